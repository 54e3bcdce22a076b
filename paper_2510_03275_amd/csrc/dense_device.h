// Device helpers of the dense operators: element types, matrix-core
// instructions, the activations and their derivatives, output conversion.
#pragma once

#include <hip/hip_runtime.h>

#include "dense.h"

namespace sdq {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// 16 x 16 products of 16-byte operands: lane l holds row l % 16 of either
// operand and the 16 bytes of depth group l / 16; accumulator v is row
// 4 (l / 16) + v of the first operand and row l % 16 of the second.
template <int ELEM> struct Elem;
template <> struct Elem<kElemF16> {
  using Scalar = _Float16;
  using Acc = f32x4;
  static constexpr int kBytes = 2;
  static __device__ inline Acc mfma(const i32x4& a, const i32x4& b, const Acc& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
template <> struct Elem<kElemBf16> {
  using Scalar = __bf16;
  using Acc = f32x4;
  static constexpr int kBytes = 2;
  static __device__ inline Acc mfma(const i32x4& a, const i32x4& b, const Acc& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                   0);
  }
};
template <> struct Elem<kElemI8> {
  using Scalar = int8_t;
  using Acc = i32x4;
  static constexpr int kBytes = 1;
  static __device__ inline Acc mfma(const i32x4& a, const i32x4& b, const Acc& c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
  }
};

// act(g) = g s(a(g)) with s the logistic function and a(g) = g (SiLU) or
// 2 sqrt(2 / pi) (g + 0.044715 g^3) (GELU's tanh form: (1 + tanh y) / 2 = s(2 y)).
// Both keep their relative accuracy where they vanish (g -> -inf).
constexpr float kGeluA = 1.5957691216057308f;        // 2 sqrt(2 / pi)
constexpr float kGeluB = 0.07135481282053126f;       // 0.044715 of it
__device__ inline float act_arg(float g, int act) {
  return act == SDQ_ACT_SILU ? g : g * (kGeluA + kGeluB * g * g);
}
__device__ inline float act_value(float g, int act) { return g / (1.0f + expf(-act_arg(g, act))); }
// act'(g) = s + g s (1 - s) a'(g); 1 - s is e^-a s, which does not cancel.
__device__ inline void act_both(float g, int act, float* value, float* slope) {
  const float e = expf(-act_arg(g, act));
  const float s = 1.0f / (1.0f + e);
  const float da = act == SDQ_ACT_SILU ? 1.0f : kGeluA + 3.0f * kGeluB * g * g;
  *value = g * s;
  // Far out either e or s has vanished and a' may be infinite: the term is zero.
  *slope = e > 0.0f && s > 0.0f ? s + g * s * (e * s) * da : s;
}

__device__ inline float load_as_float(const void* p, int64_t i, int type) {
  if (type == SDQ_F16) return static_cast<const _Float16*>(p)[i];
  if (type == SDQ_BF16) return static_cast<const __bf16*>(p)[i];
  return static_cast<const float*>(p)[i];
}
__device__ inline void store_float(void* p, int64_t i, int type, float v) {
  if (type == SDQ_F16) static_cast<_Float16*>(p)[i] = static_cast<_Float16>(v);
  else if (type == SDQ_BF16) static_cast<__bf16*>(p)[i] = static_cast<__bf16>(v);
  else static_cast<float*>(p)[i] = v;
}

// Four consecutive outputs r .. r + 3 of row i (those below cols); vector
// stores where the row length keeps every group of four aligned.
__device__ inline void store4(void* out, int64_t i, int64_t r, int64_t cols, int type, bool accumulate, f32x4 v) {
  const int64_t at = i * cols + r;
  if (r + 4 <= cols && cols % 4 == 0) {
    if (type == SDQ_F16) {
      f16x4* p = reinterpret_cast<f16x4*>(static_cast<_Float16*>(out) + at);
      if (accumulate) v += __builtin_convertvector(*p, f32x4);
      *p = __builtin_convertvector(v, f16x4);
    } else if (type == SDQ_BF16) {
      bf16x4* p = reinterpret_cast<bf16x4*>(static_cast<__bf16*>(out) + at);
      if (accumulate) v += __builtin_convertvector(*p, f32x4);
      *p = __builtin_convertvector(v, bf16x4);
    } else {
      f32x4* p = reinterpret_cast<f32x4*>(static_cast<float*>(out) + at);
      if (accumulate) v += *p;
      *p = v;
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (r + j < cols) store_float(out, at + j, type, accumulate ? load_as_float(out, at + j, type) + v[j] : v[j]);
}

// The sums of four outputs as floats: 8-bit sums with the scales of their row
// of tall (st) and of their rows of wide.
__device__ inline f32x4 scaled4(const f32x4& a, float, const float*, int64_t, int64_t) { return a; }
__device__ inline f32x4 scaled4(const i32x4& a, float st, const float* sw, int64_t r, int64_t cols) {
  f32x4 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = static_cast<float>(a[j]) * st * sw[min(r + j, cols - 1)];
  return v;
}

// Four outputs r .. r + 3 of row i from their sums (GATED: a of gate, b of up).
template <int ELEM, bool GATED>
__device__ inline void finish4(const Product& p, int z, int64_t i, int64_t r, const typename Elem<ELEM>::Acc& a,
                               const typename Elem<ELEM>::Acc& b) {
  const float st = ELEM == kElemI8 ? p.tall_scale[i] : 1.0f;
  const f32x4 g = scaled4(a, st, p.wide_scale[0], r, p.cols);
  if constexpr (!GATED) {
    store4(p.out[z], i, r, p.cols, p.out_type, p.accumulate, g);
    return;
  } else {
    const f32x4 u = scaled4(b, st, p.wide_scale[1], r, p.cols);
    f32x4 h;
#pragma unroll
    for (int v = 0; v < 4; ++v) h[v] = act_value(g[v], p.act) * u[v];
    store4(p.out[0], i, r, p.cols, p.out_type, false, h);
    if (p.g_out) {
      store4(p.g_out, i, r, p.cols, p.elem, false, g);
      store4(p.u_out, i, r, p.cols, p.elem, false, u);
    }
  }
}

}  // namespace sdq
