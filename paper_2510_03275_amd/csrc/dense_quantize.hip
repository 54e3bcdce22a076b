// 8-bit rows: per row the scale s = max(a c, 2^-126) of its largest
// magnitude a (c = fp32(1 / 127); one rounding), then q = x / s rounded to nearest, ties to
// even, of the exact quotient.  A row that holds a NaN or an infinity gets the
// scale NaN and zero codes, so that everything computed from it is NaN.
//
// The quotient is not formed: q0 = rint(x / s by the reciprocal) is at most one
// off, and where |x / s - q0| comes within 2^-12 of a half, the remainder
// x - q0 s decides.  It is exact in fp32 (one fused multiply-add): for q0 = 0
// it is x; for |q0| = 1, x is within a factor of two of s; beyond, x is a
// multiple of s's last place and the remainder below s.
#include <hip/hip_runtime.h>

#include "dense_device.h"

namespace sdq {
namespace {

__device__ inline int quantized(float x, float s, float inv) {
  const float t = x * inv;
  float q = rintf(t);
  if (fabsf(t - q) > 0.5f - 0x1p-12f) {
    const float r = __builtin_fmaf(-q, s, x);      // exact
    const float half = 0.5f * s;                   // exact: s >= 2^-126, subnormals are kept
    if (r > half || (r == half && fmodf(q, 2.0f) != 0.0f)) q += 1.0f;
    else if (r < -half || (r == -half && fmodf(q, 2.0f) != 0.0f)) q -= 1.0f;
  }
  return static_cast<int>(q);
}

template <class S>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const S* __restrict__ x, int64_t k, int8_t* __restrict__ q,
                                                            int64_t ld, float* __restrict__ scales) {
  constexpr int kPer = 16 / sizeof(S);
  __shared__ float part[4];
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x;
  const S* src = x + row * k;
  int8_t* dst = q + row * ld;
  const int64_t whole = k / kPer * kPer;
  float a = 0.0f;
  for (int64_t c = tid * kPer; c < whole; c += 256 * kPer) {
    S v[kPer];
    __builtin_memcpy(v, src + c, 16);
#pragma unroll
    for (int j = 0; j < kPer; ++j) a = __builtin_elementwise_maximum(a, fabsf(static_cast<float>(v[j])));   // NaN stays
  }
  if (whole + tid < k) a = __builtin_elementwise_maximum(a, fabsf(static_cast<float>(src[whole + tid])));
#pragma unroll
  for (int off = 32; off > 0; off /= 2) a = __builtin_elementwise_maximum(a, __shfl_xor(a, off, 64));
  if (tid % 64 == 0) part[tid / 64] = a;
  __syncthreads();
  a = __builtin_elementwise_maximum(__builtin_elementwise_maximum(part[0], part[1]),
                                    __builtin_elementwise_maximum(part[2], part[3]));
  const bool finite = a <= 3.4028234663852886e38f;
  const float s = fmaxf(a * (1.0f / 127.0f), 0x1p-126f);
  const float inv = 1.0f / s;
  if (tid == 0) scales[row] = finite ? s : __builtin_nanf("");
  for (int64_t c = tid * kPer; c < whole; c += 256 * kPer) {
    S v[kPer];
    int8_t o[kPer];
    __builtin_memcpy(v, src + c, 16);
#pragma unroll
    for (int j = 0; j < kPer; ++j) o[j] = finite ? static_cast<int8_t>(quantized(static_cast<float>(v[j]), s, inv)) : 0;
    __builtin_memcpy(dst + c, o, kPer);
  }
  if (whole + tid < k)
    dst[whole + tid] = finite ? static_cast<int8_t>(quantized(static_cast<float>(src[whole + tid]), s, inv)) : 0;
  if (k + tid < ld) dst[k + tid] = 0;      // ld - k < 16
}

}  // namespace

sdq_status launch_int8_quantize(const void* x, sdq_dtype xt, int64_t m, int64_t k, int8_t* q, int64_t ld,
                                float* scales, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(m));
  if (xt == SDQ_F16)
    quantize_rows_kernel<<<grid, 256, 0, stream>>>(static_cast<const _Float16*>(x), k, q, ld, scales);
  else if (xt == SDQ_BF16)
    quantize_rows_kernel<<<grid, 256, 0, stream>>>(static_cast<const __bf16*>(x), k, q, ld, scales);
  else
    quantize_rows_kernel<<<grid, 256, 0, stream>>>(static_cast<const float*>(x), k, q, ld, scales);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SDQ_OK : hip_error(e, "int8 quantize launch");
}

}  // namespace sdq
