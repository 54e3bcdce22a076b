// Device helpers of the 8-bit rows: the largest magnitude of a row and the codes
// of its elements (dense_quantize.hip for whole rows, dense_few.hip for its own).
//
// The quotient is not formed: q0 is x times the reciprocal of s, rounded by adding 1.5 2^23 (whose sum
// holds q0 in its low bits), at most one off; where x / s - q0 comes within 2^-12 of a half, the remainder
// x - q0 s decides.  It is exact in fp32 (one fused multiply-add): for q0 = 0
// it is x; for |q0| = 1, x is within a factor of two of s; beyond, x is a
// multiple of s's last place and the remainder below s.
#pragma once

#include "dense_device.h"

namespace sdq {

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

constexpr float kLargestFloat = 3.4028234663852886e38f;
__device__ inline float row_scale(float top) { return fmaxf(top * (1.0f / 127.0f), 0x1p-126f); }

// The 16 bytes of a row's elements as codes, four to a word.
template <class S>
__device__ inline void quantize_chunk(const u32x4& v, float s, float inv, uint32_t* o) {
  constexpr int kPer = 16 / sizeof(S);
  S e[kPer];
  __builtin_memcpy(e, &v, 16);
#pragma unroll
  for (int j = 0; j < kPer / 4; ++j) {
    float f[4];
#pragma unroll
    for (int l = 0; l < 4; ++l) f[l] = static_cast<float>(e[4 * j + l]);
    o[j] = quantize4(f, s, inv);
  }
}

}  // namespace sdq
