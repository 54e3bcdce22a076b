// The products of the dense operators for at most 16 rows (token generation):
// the weights are read once and everything else is small, so the stream of the
// weights bounds it.
//
// A workgroup forms 16 columns of every row (of a gated product, 16 of gate and
// the same 16 of up; else 16 or 32), its waves each a contiguous part of the
// depth; their sums are joined through LDS in the waves' order, so results do
// not depend on timing and need no second launch.  A wave reads its weights from memory into
// the matrix-core operand registers (lane l: row l % 16, 16 bytes at l / 16 of a
// 64-byte step), kDeep steps ahead of the products; the activations come from L2
// the same way, rows past the last as copies of it whose outputs are not
// stored.  Rows need not start aligned: only the bytes behind the last whole
// step are read element by element.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "dense_device.h"

namespace sdq {
namespace {

constexpr int kDeep = 4;      // steps of 64 bytes in flight per buffer

template <int ELEM, bool GATED, int TILES, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void few_kernel(Product p) {
  using E = Elem<ELEM>;
  using S = typename E::Scalar;
  using Acc = typename E::Acc;
  constexpr int kPer = 16 / E::kBytes, kStep = 64 / E::kBytes;
  __shared__ Acc part[WAVES][TILES][64];
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int64_t col0 = static_cast<int64_t>(blockIdx.x) * (GATED ? 16 : 16 * TILES);
  const int64_t i = lane % 16, c = (lane / 16) * kPer;
  const S* x = static_cast<const S*>(p.tall[0]) + min(i, p.rows - 1) * p.ld_tall + c;
  const S* w[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t)
    w[t] = static_cast<const S*>(p.wide[GATED ? t : 0]) + min(col0 + (GATED ? 0 : 16 * t) + i, p.cols - 1) * p.ld_wide +
           c;
  const int full = static_cast<int>(p.depth / kStep);
  const int each = (full + WAVES - 1) / WAVES;
  const int s0 = min(wave * each, full), s1 = min(s0 + each, full);

  Acc acc[TILES] = {};
  i32x4 wv[2][kDeep][TILES], xv[2][kDeep];
  auto fetch = [&](int b, int s) {      // kDeep steps from s on; steps past the end repeat the last one
#pragma unroll
    for (int d = 0; d < kDeep; ++d) {
      const int64_t at = static_cast<int64_t>(min(s + d, s1 - 1)) * kStep;
#pragma unroll
      for (int t = 0; t < TILES; ++t) __builtin_memcpy(&wv[b][d][t], w[t] + at, 16);
      __builtin_memcpy(&xv[b][d], x + at, 16);
    }
  };
  auto multiply = [&](int b, int s) {
#pragma unroll
    for (int d = 0; d < kDeep; ++d)
      if (s + d < s1)
#pragma unroll
        for (int t = 0; t < TILES; ++t) acc[t] = E::mfma(wv[b][d][t], xv[b][d], acc[t]);
  };
  if (s0 < s1) {
    fetch(0, s0);
    for (int s = s0; s < s1; s += 2 * kDeep) {
      fetch(1, s + kDeep);
      multiply(0, s);
      fetch(0, s + 2 * kDeep);
      multiply(1, s + kDeep);
    }
  }
  if (wave == WAVES - 1 && full * static_cast<int64_t>(kStep) < p.depth) {
    const int64_t at = full * static_cast<int64_t>(kStep);
    S xe[kPer], we[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) xe[j] = at + c + j < p.depth ? x[at + j] : S(0);
    i32x4 xt, wt;
    __builtin_memcpy(&xt, xe, 16);
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) we[j] = at + c + j < p.depth ? w[t][at + j] : S(0);
      __builtin_memcpy(&wt, we, 16);
      acc[t] = E::mfma(wt, xt, acc[t]);
    }
  }

#pragma unroll
  for (int t = 0; t < TILES; ++t) part[wave][t][lane] = acc[t];
  __syncthreads();
  if (wave >= (GATED ? 1 : TILES)) return;
  auto joined = [&](int t) {
    Acc sum = part[0][t][lane];
#pragma unroll
    for (int v = 1; v < WAVES; ++v) sum += part[v][t][lane];
    return sum;
  };
  const int64_t row = lane % 16, r = col0 + (GATED ? 0 : 16 * wave) + 4 * (lane / 16);
  if (row >= p.rows || r >= p.cols) return;
  const float st = ELEM == kElemI8 ? p.tall_scale[row] : 1.0f;
  if constexpr (GATED) {
    const f32x4 g = scaled4(joined(0), st, p.wide_scale[0], r, p.cols);
    const f32x4 u = scaled4(joined(1), st, p.wide_scale[1], r, p.cols);
    f32x4 h;
#pragma unroll
    for (int v = 0; v < 4; ++v) h[v] = act_value(g[v], p.act) * u[v];
    store4(p.out[0], row, r, p.cols, p.out_type, false, h);
    if (p.g_out) {
      store4(p.g_out, row, r, p.cols, p.elem, false, g);
      store4(p.u_out, row, r, p.cols, p.elem, false, u);
    }
  } else {
    store4(p.out[0], row, r, p.cols, p.out_type, p.accumulate, scaled4(joined(wave), st, p.wide_scale[0], r, p.cols));
  }
}

template <int ELEM, bool GATED, int TILES>
void launch_waves(const Product& p, hipStream_t stream) {
  const int64_t per = GATED ? 16 : 16 * TILES;
  const dim3 grid(static_cast<unsigned>((p.cols + per - 1) / per));
  // Waves enough for eight per compute unit in all, each with a whole buffer of steps at least.
  const int64_t steps = p.depth * Elem<ELEM>::kBytes / 64, units = device_compute_units();
  if (grid.x * 4 >= 8 * units || steps < 4 * kDeep) few_kernel<ELEM, GATED, TILES, 4><<<grid, 256, 0, stream>>>(p);
  else if (grid.x * 8 >= 8 * units || steps < 16 * kDeep) few_kernel<ELEM, GATED, TILES, 8><<<grid, 512, 0, stream>>>(p);
  else few_kernel<ELEM, GATED, TILES, 16><<<grid, 1024, 0, stream>>>(p);
}

}  // namespace

void launch_few(const Product& p, hipStream_t stream) {
  if (p.gated) {
    if (p.elem == kElemF16) launch_waves<kElemF16, true, 2>(p, stream);
    else if (p.elem == kElemBf16) launch_waves<kElemBf16, true, 2>(p, stream);
    else launch_waves<kElemI8, true, 2>(p, stream);
  } else {
    launch_waves<kElemI8, false, 1>(p, stream);
  }
}

}  // namespace sdq
