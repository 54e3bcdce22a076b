// The products of the dense operators on tiles of 256 rows of wide by 256, 128
// or 64 rows of tall (dense.h), for operands whose rows start 16-byte aligned.
//
// What bounds it, at 256 x 256: a step of 128 bytes of depth takes 64 matrix-core
// instructions per wave (two waves per SIMD: 2048 clocks per step), 192 KB of LDS
// reads (1536 clocks at 128 bytes) and 64 KB of copies into LDS.  So the
// matrix cores and LDS have to run side by side, and nothing may wait for memory:
//
//   tile      Eight waves; wave (wt, ww) multiplies rows 64 wt .. of both 128-row
//             halves of tall (A0, A1) with rows 32 ww .. of both halves of wide
//             (B0, B1): 128 x 64 outputs in 128 registers.  Of a gated product B0 is
//             gate and B1 the same 128 rows of up, so a lane ends with g and u of
//             the same outputs.
//   phases    A step is four phases: read A0, multiply A0 B0; read B1, A0 B1; read
//             A1, A1 B0; read the next step's B0, A1 B1.  Each phase is a reading
//             part, a barrier, 16 matrix-core instructions, a barrier.  Waves 4-7
//             run half a phase behind waves 0-3 (one barrier more before, one less
//             after), so one half of the workgroup reads LDS while the other
//             multiplies.
//   copies    Two steps sit in LDS.  A quarter (A0, A1, B0 or B1, 16 KB) is read in
//             one phase and refilled with the step after next in the phase that
//             follows: straight from memory to LDS, two 1 KB copies per wave.
//             Every phase ends with a wait for all but the last 12 copies, which
//             is the quarter read next: copies have six phases to arrive.
//   layout    Depth-contiguous operands: LDS rows of 128 bytes whose 16-byte chunk q
//             lies at q ^ (row % 8) (the copy permutes its source addresses; LDS
//             addresses of a copy are linear), so that eight lanes' reads of eight
//             rows cover all banks.  Strided operands: LDS rows of one depth (128
//             elements); a group of 16 lanes reads 4 depths x 16 elements
//             transposed (ds_read_b64_tr_b16), 32-byte granule p of depth c at
//             p ^ (c % 4 + 4 (c / 8 % 2)).
//   outputs   The sums go through LDS, half a tile at a time, so that the stores are
//             whole rows and the code that scales, activates and converts exists once
//             (unrolled over a lane's 128 sums it was 130 KB of instructions, whose
//             first fetch took 20 us).
//   splits    Where the tiles are fewer than the compute units, the depth is cut and
//             the sums of every part go to the workspace; join_kernel adds them in
//             order.
//   ends      Buffer resources end with the operand: rows past its end read as
//             zeros, as do depths past its end (for depth-contiguous rows, whose
//             neighbours follow, the lanes past the end get an address out of range).
//   order     Workgroups go to the XCDs round-robin: each XCD takes a contiguous
//             range of tiles, four tiles of tall by eight of wide at a time, whose
//             operands its L2 holds for all 32.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "dense_device.h"

namespace sdq {
namespace {

typedef __attribute__((address_space(3))) void* LdsPtr;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* LdsS4;

constexpr int kWideHalf = 16384;            // bytes of half a tile's rows of wide, one step
constexpr unsigned kOut = 0x80000000u;      // an offset past every buffer
constexpr int kRsrcWord3 = 0x00020000;

constexpr int wait_counts(int vm) { return (vm & 15) | ((vm >> 4) << 14) | (7 << 4); }   // and lgkmcnt(0)

__device__ inline void barrier() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
}

// The copies of one quarter: half a tile's rows of an operand, one step after the other.
// Everything but the lane's offsets is the same for the whole wave.
struct Quarter {
  const char* src;           // the rows at the next step
  const char* second;        // the other segment's
  int64_t bytes, bytes0;     // from there to the operand's end
  int left;                  // bytes of depth left (depth-contiguous)
};

// ROWS: of a half.  A wave issues kCopies copies per step and half (of 32 rows, waves 4-7
// repeat those of waves 0-3).
template <int BYTES, bool STRIDED, int ROWS>
struct Copier {
  static_assert(!STRIDED || ROWS == 128, "strided halves hold 128 rows");
  static constexpr int kCopies = ROWS == 128 ? 2 : 1;
  int64_t step;              // bytes from one step to the next
  int depth_bytes;
  unsigned off[2];           // the lane's two source offsets
  int chunk;                 // its 16 bytes of a step (depth-contiguous)
  __device__ inline void init(int64_t ld, int64_t depth, int wave, int lane) {
    const unsigned ld_bytes = static_cast<unsigned>(ld * BYTES);
    step = STRIDED ? 64 * static_cast<int64_t>(ld_bytes) : 128;
    depth_bytes = static_cast<int>(depth * BYTES);
    if (STRIDED) {
      const int swz = (lane / 16) | ((wave / 2 % 2) << 2);
      const int r = (((lane % 16) / 2) ^ swz) * 16 + (lane % 2) * 8;
      off[0] = (4 * wave + lane / 16) * ld_bytes + 2 * r;
      off[1] = off[0] + 32 * ld_bytes;
      chunk = 0;
    } else {
      chunk = 16 * ((lane % 8) ^ (lane / 8));
      off[0] = (8 * (ROWS == 32 ? wave % 4 : wave) + lane / 8) * ld_bytes + chunk;
      off[1] = off[0] + 64 * ld_bytes;
    }
  }
  // Rows r0 .. of n rows (r0 may lie past them: nothing is read then) from step t on; steps per segment.
  __device__ inline Quarter quarter(const void* first, const void* second, int64_t r0, int64_t n, int64_t ld,
                                    int64_t depth, int t, int steps) const {
    Quarter q;
    const int64_t at = r0 * (STRIDED ? 1 : ld) * BYTES;
    q.src = static_cast<const char*>(t < steps ? first : second) + at;
    q.second = static_cast<const char*>(second) + at;
    // Rows behind a strided operand's last one belong to the next depth: they are read, and
    // their outputs not stored.
    const int64_t valid = n - r0;
    q.bytes0 = STRIDED ? (depth * ld - r0) * BYTES : (valid < ROWS ? valid : ROWS) * ld * BYTES;
    if (valid <= 0) q.bytes0 = 0;
    const int past = t < steps ? t : t - steps;
    q.src += past * step;
    q.bytes = q.bytes0 - past * step;
    q.left = depth_bytes - 128 * past;
    return q;
  }
  // The next step of q to LDS, zeros unless `read`.
  __device__ inline void copy(Quarter& q, char* lds, int wave, bool read) const {
    unsigned o0 = off[0], o1 = off[1];
    if (!STRIDED) {
      const bool past = chunk >= q.left;
      o0 = past ? kOut : o0;
      o1 = past ? kOut : o1;
    }
    const int num = !read || q.bytes <= 0 ? 0 : q.bytes < 0x7FFFFFFF ? static_cast<int>(q.bytes) : 0x7FFFFFFF;
    const __amdgpu_buffer_rsrc_t rs =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(q.src), static_cast<short>(0), num, kRsrcWord3);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (LdsPtr)(lds + (ROWS == 32 ? wave % 4 : wave) * 1024), 16, o0, 0, 0, 0);
    if (kCopies == 2) __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (LdsPtr)(lds + 8192 + wave * 1024), 16, o1, 0, 0, 0);
    q.src += step;
    q.bytes -= step;
    q.left -= 128;
  }
  __device__ inline void next_segment(Quarter& q) const {
    q.src = q.second;
    q.bytes = q.bytes0;
    q.left = depth_bytes;
  }
};

// The lane's places in a half for fragments of 16 rows from `row` on.
template <bool STRIDED>
struct Places {
  int at[STRIDED ? 4 : 2];
  __device__ inline void init(int row, int lane) {
    const int g = lane / 16, i = lane % 16;
    if (STRIDED) {
      // depth c = 32 s + 8 g + 4 e + i / 4: swizzle i / 4 + 4 (g % 2), the same for every s and e;
      // row / 16 + n is the granule of fragment n, n ^ handled by the caller's XOR below
      for (int n = 0; n < 4; ++n) {
        const int granule = (row / 16 + n) ^ ((i / 4) | ((g % 2) << 2));
        at[n] = (8 * g + i / 4) * 256 + granule * 32 + (i % 4) * 8;
      }
    } else {
      at[0] = (row + i) * 128 + ((g ^ (i % 8)) * 16);
      at[1] = (row + i) * 128 + (((g + 4) ^ (i % 8)) * 16);
    }
  }
  // Fragment n (16 rows) of depth half s.
  __device__ inline i32x4 read(const char* lds, int n, int s) const {
    if constexpr (STRIDED) {
      const char* p = lds + at[n] + s * 8192;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsS4)p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsS4)(p + 1024));
      return __builtin_bit_cast(i32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      return *reinterpret_cast<const i32x4*>(lds + at[s] + n * 2048);
    }
  }
};

constexpr int kXcds = 8;

template <int ELEM, bool WIDE_STRIDED, bool TALL_STRIDED, bool GATED, int TALL>
__global__ __launch_bounds__(512, TALL == 64 ? 4 : 2) void wide_kernel(Product p, int splits) {
  using E = Elem<ELEM>;
  using Acc = typename E::Acc;
  constexpr int kB = E::kBytes, kStep = 128 / kB;
  constexpr int kHalf = TALL / 2, kWaveRows = kHalf / 2, kFrags = kWaveRows / 16;
  constexpr int kTallHalf = kHalf * 128, kBuf = 2 * kTallHalf + 2 * kWideHalf;
  using CopyA = Copier<kB, TALL_STRIDED, kHalf>;
  using CopyB = Copier<kB, WIDE_STRIDED, 128>;
  __shared__ __attribute__((aligned(1024))) char lds[2 * kBuf];   // [step % 2][A0, A1, B0, B1]
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int ww = wave % 4, wt = wave / 4;

  // The tile.
  constexpr int kCols = GATED ? 128 : 256;
  const unsigned nw = static_cast<unsigned>((p.cols + kCols - 1) / kCols);
  const unsigned nt = static_cast<unsigned>((p.rows + TALL - 1) / TALL);
  const unsigned total = gridDim.x, id = blockIdx.x;
  const unsigned xcd = id % kXcds, per = total / kXcds, rem = total % kXcds;
  unsigned tile = xcd * per + (xcd < rem ? xcd : rem) + id / kXcds;
  const int part = __builtin_amdgcn_readfirstlane(tile / (nw * nt));     // of the batch, or of the depth
  tile -= part * (nw * nt);
  const int z = splits > 1 ? 0 : part;
  const unsigned band = tile / (4 * nw), in_band = tile - band * (4 * nw);
  const unsigned band_rows = nt - 4 * band < 4 ? nt - 4 * band : 4;
  const unsigned tw = in_band / band_rows, tt = 4 * band + (in_band - tw * band_rows);
  const int64_t row0 = static_cast<int64_t>(__builtin_amdgcn_readfirstlane(tt)) * TALL;
  const int64_t col0 = static_cast<int64_t>(__builtin_amdgcn_readfirstlane(tw)) * kCols;

  const int seg_steps = static_cast<int>((p.depth + kStep - 1) / kStep), steps = seg_steps * p.segments;
  const int each = steps / splits, more = steps % splits, at = splits > 1 ? part : 0;
  const int t0 = at * each + min(at, more), t1 = t0 + each + (at < more ? 1 : 0);

  CopyA ca;
  CopyB cb;
  ca.init(p.ld_tall, p.depth, wave, lane);
  cb.init(p.ld_wide, p.depth, wave, lane);
  Quarter qa[2], qb[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    qa[h] = ca.quarter(p.tall[p.batch > 1 ? z : 0], p.tall[1], row0 + kHalf * h, p.rows, p.ld_tall, p.depth, t0,
                       seg_steps);
    qb[h] = cb.quarter(p.wide[GATED ? h : 0], p.wide[1], GATED ? col0 : col0 + 128 * h, p.cols, p.ld_wide, p.depth, t0,
                       seg_steps);
  }

  Places<TALL_STRIDED> pa;
  Places<WIDE_STRIDED> pb;
  pa.init(kWaveRows * wt, lane);
  pb.init(32 * ww, lane);

  // Step t of half h to its place: A (tall) or B (wide).
  auto copy_a = [&](int h, int t) {
    if (t == seg_steps && t0 < seg_steps && p.segments > 1) ca.next_segment(qa[h]);
    ca.copy(qa[h], lds + ((t - t0) % 2) * kBuf + h * kTallHalf, wave, t < t1);
  };
  auto copy_b = [&](int h, int t) {
    if (t == seg_steps && t0 < seg_steps && p.segments > 1) cb.next_segment(qb[h]);
    cb.copy(qb[h], lds + ((t - t0) % 2) * kBuf + 2 * kTallHalf + h * kWideHalf, wave, t < t1);
  };

  Acc acc[2][2][kFrags][2] = {};  // [A half][B half][rows of tall / 16][rows of wide / 16]
  i32x4 a[2][kFrags][2], b[2][2][2];   // halves: [rows / 16][depth half]

#ifndef VAR
#define VAR 0
#endif
#define VPRIO (VAR & 1)
#define VILV (VAR & 2)
#define VTWO (VAR & 4)
  auto multiply = [&](int ha, int hb) {
    if (!VILV) __builtin_amdgcn_sched_barrier(0);
    if (VPRIO) __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < kFrags; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[ha][hb][i][j] = E::mfma(b[hb][j][s], a[ha][i][s], acc[ha][hb][i][j]);
    if (VPRIO) __builtin_amdgcn_s_setprio(0);
    if (VILV) {
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, kFrags / 2 ? kFrags / 2 : 1, 0);
      }
    }
    if (!VTWO) __builtin_amdgcn_sched_barrier(0);
  };
  auto read_a = [&](const char* buf, int h) {
#pragma unroll
    for (int i = 0; i < kFrags; ++i)
#pragma unroll
      for (int s = 0; s < 2; ++s) a[h][i][s] = pa.read(buf + h * kTallHalf, i, s);
  };
  auto read_b = [&](const char* buf, int h) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int s = 0; s < 2; ++s) b[h][j][s] = pb.read(buf + 2 * kTallHalf + h * kWideHalf, j, s);
  };
  // The end of a phase: what was read has arrived, and the quarter read next, of every wave.
  auto turn = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(wait_counts(6 + 3 * CopyA::kCopies));   // all but the last six quarters
    asm volatile("" ::: "memory");
    barrier();
  };

  for (int t = t0; t < t0 + 2; ++t) {
    copy_a(0, t);
    copy_b(0, t);
    copy_b(1, t);
    copy_a(1, t);
  }
  turn();
  read_a(lds, 0);
  read_b(lds, 0);
  turn();
  copy_a(0, t0 + 2);
  turn();

#if VAR & 4
  auto turn2 = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(wait_counts(4 + 2 * CopyA::kCopies));
    asm volatile("" ::: "memory");
    barrier();
  };
  for (int t = t0; t < t1; ++t) {
    const char* cur = lds + ((t - t0) % 2) * kBuf;
    const char* nxt = lds + ((t - t0 + 1) % 2) * kBuf;
    read_b(cur, 1);
    copy_b(0, t + 2);
    multiply(0, 0);
    read_a(cur, 1);
    if (t > t0) copy_a(0, t + 2);
    multiply(0, 1);
    turn2();
    read_a(nxt, 0);
    copy_b(1, t + 2);
    multiply(1, 0);
    read_b(nxt, 0);
    copy_a(1, t + 2);
    multiply(1, 1);
    turn2();
  }
#else
  for (int t = t0; t < t1; ++t) {
    const char* cur = lds + ((t - t0) % 2) * kBuf;
    const char* nxt = lds + ((t - t0 + 1) % 2) * kBuf;
    read_b(cur, 1);
    copy_b(0, t + 2);
    multiply(0, 0);
    turn();
    read_a(cur, 1);
    copy_b(1, t + 2);
    multiply(0, 1);
    turn();
    read_a(nxt, 0);
    copy_a(1, t + 2);
    multiply(1, 0);
    turn();
    read_b(nxt, 0);
    copy_a(0, t + 3);
    multiply(1, 1);
    turn();
  }
#endif
  __builtin_amdgcn_s_waitcnt(0);      // the copies past the end land before the sums take their place
  __syncthreads();

  // Sums of half a tile: [kHalf rows][64 chunks of four columns], chunk q of row r at q ^ (r % 16).
  // Chunks 0-31 are of B0, 32-63 of B1.
  Acc* sums = reinterpret_cast<Acc*>(lds);
  const int64_t ld_part = (p.cols + 3) / 4 * 4;      // of gate and of up
#pragma unroll
  for (int ha = 0; ha < 2; ++ha) {
    if (ha) __syncthreads();
#pragma unroll
    for (int hb = 0; hb < 2; ++hb)
#pragma unroll
      for (int i = 0; i < kFrags; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int r = kWaveRows * wt + 16 * i + lane % 16, q = 32 * hb + 8 * ww + 4 * j + lane / 16;
          sums[r * 64 + (q ^ (r % 16))] = acc[ha][hb][i][j];
        }
    __syncthreads();
    if (splits > 1) {
#pragma unroll 2
      for (int o = tid; o < kHalf * 64; o += 512) {
        const int r = o / 64, q = o % 64;
        const int64_t row = row0 + kHalf * ha + r, c = col0 + 4 * (GATED ? q % 32 : q);
        if (row >= p.rows || c >= p.cols) continue;
        Acc* dst = static_cast<Acc*>(p.ws) + (part * p.rows + row) * ((GATED ? 2 : 1) * ld_part / 4) +
                   (GATED ? q / 32 : 0) * (ld_part / 4) + c / 4;
        *dst = sums[r * 64 + (q ^ (r % 16))];
      }
      continue;
    }
    constexpr int kOuts = GATED ? 32 : 64;
#pragma unroll 2
    for (int o = tid; o < kHalf * kOuts; o += 512) {
      const int r = o / kOuts, q = o % kOuts;
      const int64_t row = row0 + kHalf * ha + r, c = col0 + 4 * q;
      if (row >= p.rows || c >= p.cols) continue;
      finish4<ELEM, GATED>(p, z, row, c, sums[r * 64 + (q ^ (r % 16))],
                           GATED ? sums[r * 64 + ((q + 32) ^ (r % 16))] : Acc{});
    }
  }
}

// Adds the parts of a split product in order: one thread per four outputs.
template <int ELEM, bool GATED>
__global__ __launch_bounds__(256) void join_kernel(Product p, int splits) {
  using Acc = typename Elem<ELEM>::Acc;
  const int64_t quads = (p.cols + 3) / 4, o = blockIdx.x * int64_t{256} + threadIdx.x;
  if (o >= quads * p.rows) return;
  const int64_t row = o / quads, q = o - row * quads, ld = (GATED ? 2 : 1) * quads;
  const Acc* src = static_cast<const Acc*>(p.ws) + row * ld + q;
  Acc a = {}, b = {};
  for (int s = 0; s < splits; ++s) {
    a += src[s * p.rows * ld];
    if (GATED) b += src[s * p.rows * ld + quads];
  }
  finish4<ELEM, GATED>(p, 0, row, 4 * q, a, b);
}

template <int ELEM, bool WS, bool TS, bool GATED, int TALL>
void launch_tiles(const Product& p, int splits, hipStream_t stream) {
  const int64_t per = GATED ? 128 : 256;
  const int64_t tiles = (p.cols + per - 1) / per * ((p.rows + TALL - 1) / TALL);
  wide_kernel<ELEM, WS, TS, GATED, TALL>
      <<<dim3(static_cast<unsigned>(tiles * p.batch * splits)), 512, 0, stream>>>(p, splits);
  if (splits > 1) {
    const int64_t quads = (p.cols + 3) / 4 * p.rows;
    join_kernel<ELEM, GATED><<<dim3(static_cast<unsigned>((quads + 255) / 256)), 256, 0, stream>>>(p, splits);
  }
}

template <int ELEM, bool WS, bool GATED>
void launch_tall(const Product& p, const WidePlan& plan, hipStream_t stream) {
  if (plan.tall == 64) launch_tiles<ELEM, WS, false, GATED, 64>(p, plan.splits, stream);
  else if (plan.tall == 128) launch_tiles<ELEM, WS, false, GATED, 128>(p, plan.splits, stream);
  else launch_tiles<ELEM, WS, false, GATED, 256>(p, plan.splits, stream);
}

template <int ELEM>
void launch_elem(const Product& p, const WidePlan& plan, hipStream_t stream) {
  if (p.gated) return launch_tall<ELEM, false, true>(p, plan, stream);
  if constexpr (ELEM == kElemI8) launch_tall<ELEM, false, false>(p, plan, stream);
  else if (p.tall_strided) launch_tiles<ELEM, true, true, false, 256>(p, plan.splits, stream);
  else launch_tall<ELEM, true, false>(p, plan, stream);
}

}  // namespace

size_t wide_part_bytes(const Product& p, int splits) {
  return splits > 1 ? static_cast<size_t>(p.rows) * ((p.cols + 3) / 4) * 16 * (p.gated ? 2 : 1) * splits : 0;
}

WidePlan wide_plan(const Product& p) {
  const int64_t bytes = p.elem == kElemI8 ? 1 : 2;
  const int64_t steps = (p.depth * bytes + 127) / 128 * p.segments, units = device_compute_units();
  const int64_t col_tiles = (p.cols + (p.gated ? 127 : 255)) / (p.gated ? 128 : 256);
  WidePlan best;
  double best_us = 0;
  for (int tall = 256; tall >= (p.tall_strided ? 256 : 64); tall /= 2) {
    const int64_t tiles = col_tiles * ((p.rows + tall - 1) / tall) * p.batch;
    const int64_t at_once = tall == 64 ? 2 * units : units;
    const double step_us = tall == 256 ? 0.95 : tall == 128 ? 0.6 : 0.9, fixed_us = tall == 256 ? 6 : 4;
    for (int splits = 1; splits <= (p.batch > 1 ? 1 : 32) && (splits == 1 || steps / splits >= 4); ++splits) {
      const int64_t turns = (tiles * splits + at_once - 1) / at_once;
      const double us = turns * (fixed_us + ((steps + splits - 1) / splits) * step_us) +
                        (splits > 1 ? 3.0 + wide_part_bytes(p, splits) * 2e-6 / 4.0 : 0.0);
      if (best.splits == 0 || us < best_us) {
        best.tall = tall;
        best.splits = splits;
        best_us = us;
      }
    }
  }
  return best;
}

void launch_wide(const Product& p, hipStream_t stream) {
  WidePlan plan = wide_plan(p);
  if (const char* f = getenv("WIDE_FORCE")) sscanf(f, "%d,%d", &plan.tall, &plan.splits);
  while (plan.splits > 1 && wide_part_bytes(p, plan.splits) > p.ws_bytes) --plan.splits;
  if (plan.tall == 256) {
    launch_big(p, plan.splits, stream);
    if (plan.splits > 1) {
      const int64_t quads = (p.cols + 3) / 4 * p.rows;
      const dim3 grid(static_cast<unsigned>((quads + 255) / 256));
      if (p.elem == kElemI8 && p.gated) join_kernel<kElemI8, true><<<grid, 256, 0, stream>>>(p, plan.splits);
      else if (p.elem == kElemI8) join_kernel<kElemI8, false><<<grid, 256, 0, stream>>>(p, plan.splits);
      else if (p.gated) join_kernel<kElemF16, true><<<grid, 256, 0, stream>>>(p, plan.splits);
      else join_kernel<kElemF16, false><<<grid, 256, 0, stream>>>(p, plan.splits);
    }
    return;
  }
  if (p.elem == kElemF16) launch_elem<kElemF16>(p, plan, stream);
  else if (p.elem == kElemBf16) launch_elem<kElemBf16>(p, plan, stream);
  else launch_elem<kElemI8>(p, plan, stream);
}

}  // namespace sdq
