// The products of the dense operators (dense.h) on the matrix cores: fp16 and
// bf16 operands with fp32 sums, 8-bit operands with exact int32 sums.
//
// product_kernel: any sizes and alignment.  A workgroup of four waves forms a
// 64 x 64 tile, each wave 32 x 32 (2 x 2 matrix-core tiles).  Both operands go
// through registers to LDS in steps of 128 bytes of depth; c past depth and rows
// past the end are zeros in both.  Of a gated product, the 32 rows of wide that a
// wave multiplies are 16 of gate and the same 16 of up, so that one lane ends
// with g and u of the same outputs and the activation needs no exchange.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "dense_device.h"

namespace sdq {
namespace {

constexpr int kTile = 64;               // rows of either operand per workgroup
constexpr int kStepBytes = 128;         // depth per step
constexpr int kLdsRow = kStepBytes + 16;   // padded: a wave's 16-byte reads of 16 rows spread over the banks

// 16 bytes of row `row` from depth c on: zeros past the row's end and for rows past n.
template <class S>
__device__ inline i32x4 load_row_chunk(const S* __restrict__ p, int64_t ld, int64_t row, int64_t n, int64_t c,
                                       int64_t depth) {
  constexpr int kPer = 16 / sizeof(S);
  i32x4 v = {0, 0, 0, 0};
  if (row < n && c < depth) {
    const S* src = p + row * ld + c;
    if (c + kPer <= depth) {
      __builtin_memcpy(&v, src, 16);      // rows need not start aligned
    } else {
      S tmp[kPer];
#pragma unroll
      for (int j = 0; j < kPer; ++j) tmp[j] = c + j < depth ? src[j] : S(0);
      __builtin_memcpy(&v, tmp, 16);
    }
  }
  return v;
}

template <int ELEM, bool WIDE_STRIDED, bool TALL_STRIDED, bool GATED>
__global__ __launch_bounds__(256) void product_kernel(Product p) {
  using E = Elem<ELEM>;
  using S = typename E::Scalar;
  using Acc = typename E::Acc;
  constexpr int kPer = 16 / E::kBytes;            // elements per 16-byte chunk
  constexpr int kStep = kStepBytes / E::kBytes;   // elements of depth per step
  constexpr int kCols = GATED ? kTile / 2 : kTile;  // outputs per tile along cols
  __shared__ __attribute__((aligned(16))) char lds[2][kTile * kLdsRow];   // wide, tall
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int wr = wave % 2, wt = wave / 2;         // the wave's 32 rows of wide and of tall
  const int64_t nx = (p.cols + kCols - 1) / kCols, ny = (p.rows + kTile - 1) / kTile;
  const int64_t col0 = blockIdx.x % nx * kCols;
  const int64_t row0 = blockIdx.x / nx % ny * kTile;
  const int z = static_cast<int>(blockIdx.x / nx / ny);
  Acc acc[2][2] = {};

  for (int seg = 0; seg < p.segments; ++seg) {
    const S* tall = static_cast<const S*>(p.tall[p.batch > 1 ? z : seg]);
    for (int64_t c0 = 0; c0 < p.depth; c0 += kStep) {
      __syncthreads();
      for (int op = 0; op < 2; ++op) {
        char* dst = lds[op];
        const bool strided = op == 0 ? WIDE_STRIDED : TALL_STRIDED;
        const int64_t ld = op == 0 ? p.ld_wide : p.ld_tall;
        if (!strided) {
          for (int ch = tid; ch < kTile * (kStepBytes / 16); ch += 256) {
            const int r = ch / (kStepBytes / 16), q = ch % (kStepBytes / 16);
            i32x4 v;
            if (op == 0 && GATED) {
              const S* w = static_cast<const S*>(p.wide[(r % 32) / 16]);
              v = load_row_chunk(w, ld, col0 + 16 * (r / 32) + r % 16, p.cols, c0 + q * kPer, p.depth);
            } else if (op == 0) {
              v = load_row_chunk(static_cast<const S*>(p.wide[seg]), ld, col0 + r, p.cols, c0 + q * kPer, p.depth);
            } else {
              v = load_row_chunk(tall, ld, row0 + r, p.rows, c0 + q * kPer, p.depth);
            }
            *reinterpret_cast<i32x4*>(dst + r * kLdsRow + q * 16) = v;
          }
        } else {
          // r contiguous: chunks of rows, written to LDS element by element.
          const S* src = op == 0 ? static_cast<const S*>(p.wide[seg]) : tall;
          const int64_t r0 = op == 0 ? col0 : row0, n = op == 0 ? p.cols : p.rows;
          for (int ch = tid; ch < kStep * (kTile / kPer); ch += 256) {
            const int c = ch / (kTile / kPer), q = ch % (kTile / kPer);
            const i32x4 v = load_row_chunk(src, ld, c0 + c, p.depth, r0 + q * kPer, n);
            S e[kPer];
            __builtin_memcpy(e, &v, 16);
#pragma unroll
            for (int j = 0; j < kPer; ++j)
              *reinterpret_cast<S*>(dst + (q * kPer + j) * kLdsRow + c * E::kBytes) = e[j];
          }
        }
      }
      __syncthreads();
#pragma unroll
      for (int s = 0; s < kStepBytes / 64; ++s) {
        i32x4 a[2], b[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int at = 64 * s + 16 * (lane / 16);
          a[i] = *reinterpret_cast<const i32x4*>(lds[0] + (32 * wr + 16 * i + lane % 16) * kLdsRow + at);
          b[i] = *reinterpret_cast<const i32x4*>(lds[1] + (32 * wt + 16 * i + lane % 16) * kLdsRow + at);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = E::mfma(a[i], b[j], acc[i][j]);
      }
    }
  }

#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int64_t i = row0 + 32 * wt + 16 * j + lane % 16;
    if (i >= p.rows) continue;
    const float st = ELEM == kElemI8 ? p.tall_scale[i] : 1.0f;
#pragma unroll
    for (int w = 0; w < (GATED ? 1 : 2); ++w) {
      const int64_t r = col0 + (GATED ? 16 : 32) * wr + 16 * w + 4 * (lane / 16);
      if (r >= p.cols) continue;
      WideScales<ELEM, GATED> sw;
      sw.load(p, r);
      with_out_type<ELEM>(p, [&](auto type) {
        finish4<ELEM, GATED, decltype(type)::value>(p, z, i, r, acc[w][j], acc[1][j], st, sw);
      });
    }
  }
}

template <int ELEM, bool WS, bool TS, bool GATED>
void launch_tile(const Product& p, hipStream_t stream) {
  const int64_t per = GATED ? kTile / 2 : kTile;
  const int64_t tiles = (p.cols + per - 1) / per * ((p.rows + kTile - 1) / kTile) * p.batch;
  product_kernel<ELEM, WS, TS, GATED><<<dim3(static_cast<unsigned>(tiles)), 256, 0, stream>>>(p);
}

template <int ELEM>
void launch_any(const Product& p, hipStream_t stream) {
  if (p.gated) return launch_tile<ELEM, false, false, true>(p, stream);
  if constexpr (ELEM == kElemI8) {
    launch_tile<ELEM, false, false, false>(p, stream);
  } else if (p.tall_strided) {
    launch_tile<ELEM, true, true, false>(p, stream);
  } else {
    launch_tile<ELEM, true, false, false>(p, stream);
  }
}

// dg and du, eight elements per thread.
template <class S>
__global__ __launch_bounds__(256) void gate_gradient_kernel(const S* __restrict__ dh, const S* __restrict__ g,
                                                            const S* __restrict__ u, int64_t count, int act,
                                                            S* __restrict__ dg, S* __restrict__ du) {
  const int64_t i = (blockIdx.x * int64_t{256} + threadIdx.x) * 8;
  if (i >= count) return;
  S a[8], b[8], c[8], x[8], y[8];
  const int n = static_cast<int>(count - i < 8 ? count - i : 8);
  if (n == 8) {
    __builtin_memcpy(a, __builtin_assume_aligned(dh + i, 16), 16);
    __builtin_memcpy(b, __builtin_assume_aligned(g + i, 16), 16);
    __builtin_memcpy(c, __builtin_assume_aligned(u + i, 16), 16);
  } else {
    for (int j = 0; j < 8; ++j) {
      a[j] = j < n ? dh[i + j] : S(0);
      b[j] = j < n ? g[i + j] : S(0);
      c[j] = j < n ? u[i + j] : S(0);
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float value, slope;
    act_both(static_cast<float>(b[j]), act, &value, &slope);
    x[j] = static_cast<S>(static_cast<float>(a[j]) * static_cast<float>(c[j]) * slope);
    y[j] = static_cast<S>(static_cast<float>(a[j]) * value);
  }
  if (n == 8) {
    __builtin_memcpy(__builtin_assume_aligned(dg + i, 16), x, 16);
    __builtin_memcpy(__builtin_assume_aligned(du + i, 16), y, 16);
  } else {
    for (int j = 0; j < n; ++j) {
      dg[i + j] = x[j];
      du[i + j] = y[j];
    }
  }
}

}  // namespace

// Whether every 16 bytes that a tile reads of either operand lie in one row and start aligned,
// and 128 rows' offsets fit 31 bits.
static bool rows_aligned(const Product& p) {
  const int64_t b = p.elem == kElemI8 ? 1 : 2;
  if (p.ld_wide * b % 16 || p.ld_tall * b % 16) return false;
  return std::max(p.ld_wide, p.ld_tall) * b < (int64_t{1} << 23) && p.depth > 0 && p.depth <= (int64_t{1} << 29);
}

size_t product_ws_bytes(const Product& p) {
  return rows_aligned(p) ? 1 << 28 : 0;
}

sdq_status launch_product(const Product& p, hipStream_t stream) {
  if (p.rows <= (getenv("FEW") ? atoi(getenv("FEW")) : 64) && !p.wide_strided) launch_few(p, stream);
  else if (rows_aligned(p)) launch_wide(p, stream);
  else if (p.elem == kElemF16) launch_any<kElemF16>(p, stream);
  else if (p.elem == kElemBf16) launch_any<kElemBf16>(p, stream);
  else launch_any<kElemI8>(p, stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SDQ_OK : hip_error(e, "product launch");
}

sdq_status launch_gate_gradient(const void* dh, const void* g, const void* u, sdq_dtype t, int64_t count, int act,
                                void* dg, void* du, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>((count + 2047) / 2048));
  if (t == SDQ_F16)
    gate_gradient_kernel<<<grid, 256, 0, stream>>>(static_cast<const _Float16*>(dh), static_cast<const _Float16*>(g),
                                                   static_cast<const _Float16*>(u), count, act,
                                                   static_cast<_Float16*>(dg), static_cast<_Float16*>(du));
  else
    gate_gradient_kernel<<<grid, 256, 0, stream>>>(static_cast<const __bf16*>(dh), static_cast<const __bf16*>(g),
                                                   static_cast<const __bf16*>(u), count, act, static_cast<__bf16*>(dg),
                                                   static_cast<__bf16*>(du));
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SDQ_OK : hip_error(e, "gate gradient launch");
}

}  // namespace sdq
