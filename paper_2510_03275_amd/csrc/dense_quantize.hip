// 8-bit rows: per row the scale s = max(a c, 2^-126) of its largest
// magnitude a (c = fp32(1 / 127); one rounding), then q = x / s rounded to nearest, ties to
// even, of the exact quotient.  A row that holds a NaN or an infinity gets the
// scale NaN and zero codes, so that everything computed from it is NaN.
//
// The quotient is not formed: q0 is x times the reciprocal of s, rounded by adding 1.5 2^23 (whose sum
// holds q0 in its low bits), at most one off; where x / s - q0 comes within 2^-12 of a half, the remainder
// x - q0 s decides.  It is exact in fp32 (one fused multiply-add): for q0 = 0
// it is x; for |q0| = 1, x is within a factor of two of s; beyond, x is a
// multiple of s's last place and the remainder below s.
#include <hip/hip_runtime.h>

#include "dense_device.h"

namespace sdq {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The codes of four elements, one to a byte.  Six vector instructions per element of a 16-bit row in
// all (its magnitude taken as an integer, two at a time): at fifteen they bounded rows of 8192.
__device__ inline uint32_t quantize4(const float* v, float s, float inv) {
  constexpr float kRound = 12582912.0f;      // 1.5 x 2^23
  float q[4], far = 0.0f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    q[j] = __builtin_fmaf(v[j], inv, kRound);
    far = fmaxf(far, fabsf(__builtin_fmaf(v[j], inv, kRound - q[j])));
  }
  if (far > 0.5f - 0x1p-12f) {
    const float half = 0.5f * s;                   // exact: s >= 2^-126, subnormals are kept
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float r = __builtin_fmaf(kRound - q[j], s, v[j]);      // exact where it decides
      const bool odd = (__float_as_uint(q[j]) & 1u) != 0;
      if (r > half || (r == half && odd)) q[j] += 1.0f;
      else if (r < -half || (r == -half && odd)) q[j] -= 1.0f;
    }
  }
  // byte 0 of each: bytes 0-3 of the selector's numbers are of the second operand, 4-7 of the first, 12 is zero
  return __builtin_amdgcn_perm(__float_as_uint(q[1]), __float_as_uint(q[0]), 0x0C0C0400u) |
         __builtin_amdgcn_perm(__float_as_uint(q[3]), __float_as_uint(q[2]), 0x04000C0Cu);
}

// The largest magnitude of a row's chunks, as the bits of its elements (infinities and NaN above all
// numbers): fp32, or two of 16 bits side by side.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <class S>
__device__ inline uint32_t larger(uint32_t a, uint32_t bits) {
  if constexpr (sizeof(S) == 4) return max(a, bits & 0x7FFFFFFFu);
  else
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                                  __builtin_bit_cast(u16x2, bits & 0x7FFF7FFFu)));
}
template <class S>
__device__ inline float magnitude(uint32_t a) {
  if constexpr (sizeof(S) == 4) return __uint_as_float(a);
  else return static_cast<float>(__builtin_bit_cast(S, static_cast<uint16_t>(max(a & 0xFFFFu, a >> 16))));
}

// T threads to a row (a wave each of four rows, or a workgroup), which hold up to CHUNKS chunks of it
// each in registers, so that memory is read once and all of a row's reads are in flight together;
// the chunks of a longer row behind those are read twice.  Bound by memory: 1.17 GB of fp32 weights
// in rows of 28672 take 214-219 us (5.4 TB/s, a large copy's rate), 4096 rows of 8192 bf16 20 us (4.9 TB/s), one row of 4096 3 us (latency).
//   A chunk that would reach past the row's end starts earlier and shares elements with the one before
// it: both threads find the same codes.  Rows shorter than a chunk go element by element.
template <class S, int T, int CHUNKS>
__global__ __launch_bounds__(T == 64 ? 256 : T) void quantize_rows_kernel(const S* __restrict__ x, int64_t m, int64_t k,
                                                                          int8_t* __restrict__ q, int64_t ld,
                                                                          float* __restrict__ scales) {
  constexpr int kPer = 16 / sizeof(S);
  __shared__ uint32_t part[T / 64];
  const int64_t row = T == 64 ? blockIdx.x * int64_t{4} + threadIdx.x / 64 : blockIdx.x;
  if (row >= m) return;
  const int tid = threadIdx.x % T;
  const S* src = x + row * k;      // rows need not start aligned
  int8_t* dst = q + row * ld;
  const int64_t chunks = (k + kPer - 1) / kPer, last = k - kPer;
  auto load = [&](int64_t c) {      // chunks past the end: the last one once more
    u32x4 v;
    if (last >= 0) {
      __builtin_memcpy(&v, src + min(c * kPer, last), 16);
    } else {
      S e[kPer];
#pragma unroll
      for (int j = 0; j < kPer; ++j) e[j] = j < k ? src[j] : S(0);
      __builtin_memcpy(&v, e, 16);
    }
    return v;
  };
  auto largest = [](const u32x4& v, uint32_t a) {
#pragma unroll
    for (int j = 0; j < 4; ++j) a = larger<S>(a, v[j]);
    return a;
  };
  u32x4 v[CHUNKS];
#pragma unroll
  for (int j = 0; j < CHUNKS; ++j) v[j] = load(tid + T * j);
  uint32_t a = 0;
#pragma unroll
  for (int j = 0; j < CHUNKS; ++j) a = largest(v[j], a);
  for (int64_t c = tid + T * CHUNKS; c < chunks; c += T) a = largest(load(c), a);
#pragma unroll
  for (int off = 32; off > 0; off /= 2) a = larger<S>(a, __shfl_xor(a, off, 64));
  if (T > 64) {
    if (tid % 64 == 0) part[tid / 64] = a;
    __syncthreads();
    a = part[0];
#pragma unroll
    for (int w = 1; w < T / 64; ++w) a = larger<S>(a, part[w]);
  }
  const float top = magnitude<S>(a);
  const bool finite = top <= 3.4028234663852886e38f;
  const float s = fmaxf(top * (1.0f / 127.0f), 0x1p-126f);
  const float inv = 1.0f / s;
  if (tid == 0) scales[row] = finite ? s : __builtin_nanf("");
  auto store = [&](int64_t c, const u32x4& w) {
    if (c >= chunks) return;
    S e[kPer];
    __builtin_memcpy(e, &w, 16);
    uint32_t o[kPer / 4] = {};
    if (finite)
#pragma unroll
      for (int j = 0; j < kPer / 4; ++j) {
        float f[4];
#pragma unroll
        for (int l = 0; l < 4; ++l) f[l] = static_cast<float>(e[4 * j + l]);
        o[j] = quantize4(f, s, inv);
      }
    if (last >= 0) {
      __builtin_memcpy(dst + min(c * kPer, last), o, kPer);
    } else {
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (j < k) dst[j] = static_cast<int8_t>(o[j / 4] >> (8 * (j % 4)));
    }
  };
#pragma unroll
  for (int j = 0; j < CHUNKS; ++j) store(tid + T * j, v[j]);
  for (int64_t c = tid + T * CHUNKS; c < chunks; c += T) store(c, load(c));
  if (k + tid < ld) dst[k + tid] = 0;      // ld - k < 16
}

// The fewest threads whose registers hold a row in four chunks each; of few rows more threads.
template <class S>
void launch_rows(const S* x, int64_t m, int64_t k, int8_t* q, int64_t ld, float* scales, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(m));
  const int64_t chunks = (k + 16 / sizeof(S) - 1) / (16 / sizeof(S)), wide = m <= device_compute_units() ? 4 : 1;
  if (chunks * wide <= 64 * 2)
    quantize_rows_kernel<S, 64, 2><<<dim3(static_cast<unsigned>((m + 3) / 4)), 256, 0, stream>>>(x, m, k, q, ld, scales);
  else if (chunks * wide <= 256 * 4) quantize_rows_kernel<S, 256, 4><<<grid, 256, 0, stream>>>(x, m, k, q, ld, scales);
  else if (chunks * wide <= 512 * 4) quantize_rows_kernel<S, 512, 4><<<grid, 512, 0, stream>>>(x, m, k, q, ld, scales);
  else if (chunks <= 1024 * 4) quantize_rows_kernel<S, 1024, 4><<<grid, 1024, 0, stream>>>(x, m, k, q, ld, scales);
  else quantize_rows_kernel<S, 1024, 8><<<grid, 1024, 0, stream>>>(x, m, k, q, ld, scales);
}

}  // namespace

sdq_status launch_int8_quantize(const void* x, sdq_dtype xt, int64_t m, int64_t k, int8_t* q, int64_t ld,
                                float* scales, hipStream_t stream) {
  if (xt == SDQ_F16) launch_rows(static_cast<const _Float16*>(x), m, k, q, ld, scales, stream);
  else if (xt == SDQ_BF16) launch_rows(static_cast<const __bf16*>(x), m, k, q, ld, scales, stream);
  else launch_rows(static_cast<const float*>(x), m, k, q, ld, scales, stream);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SDQ_OK : hip_error(e, "int8 quantize launch");
}

}  // namespace sdq
