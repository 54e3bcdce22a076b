// 8-bit rows: per row the scale s = max(a c, 2^-126) of its largest
// magnitude a (c = fp32(1 / 127); one rounding), then q = x / s rounded to nearest, ties to
// even, of the exact quotient.  A row that holds a NaN or an infinity gets the
// scale NaN and zero codes, so that everything computed from it is NaN.
//
#include <hip/hip_runtime.h>

#include "dense_quantize.h"

namespace sdq {
namespace {

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
  constexpr int kRows = T == 64 ? 4 : 1;      // of a workgroup
  const int tid = threadIdx.x % T;
  for (int64_t row = blockIdx.x * int64_t{kRows} + threadIdx.x / T; row < m; row += gridDim.x * int64_t{kRows}) {
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
    const bool finite = top <= kLargestFloat;
    const float s = row_scale(top);
    const float inv = 1.0f / s;
    if (tid == 0) scales[row] = finite ? s : __builtin_nanf("");
    auto store = [&](int64_t c, const u32x4& w) {
      if (c >= chunks) return;
      uint32_t o[kPer / 4] = {};
      if (finite) quantize_chunk<S>(w, s, inv, o);
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
    for (int64_t c = k + tid; c < ld; c += T) dst[c] = 0;
    if (T > 64) __syncthreads();             // part is read before the next row's
  }
}

// The fewest threads whose registers hold a row in four chunks each; of few rows more threads.
template <class S>
void launch_rows(const S* x, int64_t m, int64_t k, int8_t* q, int64_t ld, float* scales, hipStream_t stream) {
  constexpr int64_t kMost = int64_t{1} << 20;      // workgroups: their threads are counted in 32 bits
  const dim3 grid(static_cast<unsigned>(m < kMost ? m : kMost)), grid4(static_cast<unsigned>(m < 4 * kMost ? (m + 3) / 4 : kMost));
  const int64_t chunks = (k + 16 / sizeof(S) - 1) / (16 / sizeof(S)), wide = m <= device_compute_units() ? 4 : 1;
  if (chunks * wide <= 64 * 2)
    quantize_rows_kernel<S, 64, 2><<<grid4, 256, 0, stream>>>(x, m, k, q, ld, scales);
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
