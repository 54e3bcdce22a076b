// The products of the dense operators on 256 x 256 tiles (dense.h), for operands
// whose rows start 16-byte aligned.
//
// What bounds it: a step of 128 bytes of depth takes 64 matrix-core
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

constexpr int kQuarter = 16384, kHalfRows = 128, kBuf = 4 * kQuarter;
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

template <int BYTES, bool STRIDED>
struct Copier {
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
      off[0] = (8 * wave + lane / 8) * ld_bytes + chunk;
      off[1] = off[0] + 64 * ld_bytes;
    }
  }
  // Rows r0 .. of n rows (r0 may lie past them: nothing is read then).
  __device__ inline Quarter quarter(const void* first, const void* second, int64_t r0, int64_t n, int64_t ld,
                                    int64_t depth) const {
    Quarter q;
    const int64_t at = r0 * (STRIDED ? 1 : ld) * BYTES;
    q.src = static_cast<const char*>(first) + at;
    q.second = static_cast<const char*>(second) + at;
    // Rows behind a strided operand's last one belong to the next depth: they are read, and
    // their outputs not stored.
    const int64_t valid = n - r0;
    q.bytes0 = STRIDED ? ((depth - 1) * ld + valid) * BYTES : (valid < kHalfRows ? valid : kHalfRows) * ld * BYTES;
    if (valid <= 0) q.bytes0 = 0;
    q.bytes = q.bytes0;
    q.left = depth_bytes;
    return q;
  }
  // The next step of q to LDS.  Past the last one the offsets are out of range: zeros.
  __device__ inline void copy(Quarter& q, char* lds, int wave) const {
    unsigned o0 = off[0], o1 = off[1];
    if (!STRIDED) {
      const bool past = chunk >= q.left;
      o0 = past ? kOut : o0;
      o1 = past ? kOut : o1;
    }
    const int num = q.bytes <= 0 ? 0 : q.bytes < 0x7FFFFFFF ? static_cast<int>(q.bytes) : 0x7FFFFFFF;
    const __amdgpu_buffer_rsrc_t rs =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(q.src), static_cast<short>(0), num, kRsrcWord3);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (LdsPtr)(lds + wave * 1024), 16, o0, 0, 0, 0);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (LdsPtr)(lds + 8192 + wave * 1024), 16, o1, 0, 0, 0);
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

template <int ELEM, bool WIDE_STRIDED, bool TALL_STRIDED, bool GATED>
__global__ __launch_bounds__(512, 2) void wide_kernel(Product p) {
  using E = Elem<ELEM>;
  using Acc = typename E::Acc;
  constexpr int kB = E::kBytes, kStep = 128 / kB;
  __shared__ __attribute__((aligned(1024))) char lds[2 * kBuf];   // [step % 2][A0, A1, B0, B1]
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int ww = wave % 4, wt = wave / 4;

  // The tile.
  constexpr int kCols = GATED ? 128 : 256;
  const unsigned nw = static_cast<unsigned>((p.cols + kCols - 1) / kCols);
  const unsigned nt = static_cast<unsigned>((p.rows + 255) / 256);
  const unsigned total = gridDim.x, id = blockIdx.x;
  const unsigned xcd = id % kXcds, per = total / kXcds, rem = total % kXcds;
  unsigned tile = xcd * per + (xcd < rem ? xcd : rem) + id / kXcds;
  const int z = __builtin_amdgcn_readfirstlane(tile / (nw * nt));
  tile -= z * (nw * nt);
  const unsigned band = tile / (4 * nw), in_band = tile - band * (4 * nw);
  const unsigned band_rows = nt - 4 * band < 4 ? nt - 4 * band : 4;
  const unsigned tw = in_band / band_rows, tt = 4 * band + (in_band - tw * band_rows);
  const int64_t row0 = static_cast<int64_t>(__builtin_amdgcn_readfirstlane(tt)) * 256;
  const int64_t col0 = static_cast<int64_t>(__builtin_amdgcn_readfirstlane(tw)) * kCols;

  Copier<kB, TALL_STRIDED> ca;
  Copier<kB, WIDE_STRIDED> cb;
  ca.init(p.ld_tall, p.depth, wave, lane);
  cb.init(p.ld_wide, p.depth, wave, lane);
  Quarter qa[2], qb[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    qa[h] = ca.quarter(p.tall[p.batch > 1 ? z : 0], p.tall[1], row0 + kHalfRows * h, p.rows, p.ld_tall, p.depth);
    qb[h] = cb.quarter(p.wide[GATED ? h : 0], p.wide[1], GATED ? col0 : col0 + kHalfRows * h, p.cols, p.ld_wide,
                       p.depth);
  }
  const int seg_steps = static_cast<int>((p.depth + kStep - 1) / kStep), steps = seg_steps * p.segments;

  Places<TALL_STRIDED> pa;
  Places<WIDE_STRIDED> pb;
  pa.init(64 * wt, lane);
  pb.init(32 * ww, lane);

  // Step t of half h to its place: A (tall) or B (wide).
  auto copy_a = [&](int h, int t) {
    if (t == seg_steps && p.segments > 1) ca.next_segment(qa[h]);
    ca.copy(qa[h], lds + (t % 2) * kBuf + h * kQuarter, wave);
  };
  auto copy_b = [&](int h, int t) {
    if (t == seg_steps && p.segments > 1) cb.next_segment(qb[h]);
    cb.copy(qb[h], lds + (t % 2) * kBuf + (2 + h) * kQuarter, wave);
  };

  Acc acc[2][2][4][2] = {};       // [A half][B half][rows of tall / 16][rows of wide / 16]
  i32x4 a[4][2], b[2][2][2];      // A half: [rows / 16][depth half]; B: [half][rows / 16][depth half]

  auto multiply = [&](int ha, int hb) {
    barrier();
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[ha][hb][i][j] = E::mfma(b[hb][j][s], a[i][s], acc[ha][hb][i][j]);
    __builtin_amdgcn_s_setprio(0);
    barrier();
  };
  auto read_a = [&](const char* q) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int s = 0; s < 2; ++s) a[i][s] = pa.read(q, i, s);
  };
  auto read_b = [&](const char* q, int h) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int s = 0; s < 2; ++s) b[h][j][s] = pb.read(q, j, s);
  };
  auto wait = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(wait_counts(12));
    asm volatile("" ::: "memory");
  };

  for (int t = 0; t < 2; ++t) {
    copy_b(0, t);
    copy_a(0, t);
    copy_b(1, t);
    copy_a(1, t);
  }
  wait();
  barrier();
  read_b(lds + 2 * kQuarter, 0);
  wait();
  barrier();
  if (wt == 1) barrier();

  for (int t = 0; t < steps; ++t) {
    const char* cur = lds + (t % 2) * kBuf;
    const char* nxt = lds + ((t + 1) % 2) * kBuf;
    read_a(cur);
    copy_b(0, t + 2);
    wait();
    multiply(0, 0);
    read_b(cur + 3 * kQuarter, 1);
    copy_a(0, t + 2);
    wait();
    multiply(0, 1);
    read_a(cur + kQuarter);
    copy_b(1, t + 2);
    wait();
    multiply(1, 0);
    read_b(nxt + 2 * kQuarter, 0);
    copy_a(1, t + 2);
    wait();
    multiply(1, 1);
  }
  if (wt == 0) barrier();
  __builtin_amdgcn_s_waitcnt(0);      // no copy lands after the workgroup's LDS is released

#pragma unroll
  for (int ha = 0; ha < 2; ++ha)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t row = row0 + kHalfRows * ha + 64 * wt + 16 * i + lane % 16;
      if (row >= p.rows) continue;
      const float st = ELEM == kElemI8 ? p.tall_scale[row] : 1.0f;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int64_t r0 = col0 + 32 * ww + 16 * j + 4 * (lane / 16);
        if constexpr (GATED) {
          if (r0 >= p.cols) continue;
          const f32x4 g = scaled4(acc[ha][0][i][j], st, p.wide_scale[0], r0, p.cols);
          const f32x4 u = scaled4(acc[ha][1][i][j], st, p.wide_scale[1], r0, p.cols);
          f32x4 h;
#pragma unroll
          for (int v = 0; v < 4; ++v) h[v] = act_value(g[v], p.act) * u[v];
          store4(p.out[0], row, r0, p.cols, p.out_type, false, h);
          if (p.g_out) {
            store4(p.g_out, row, r0, p.cols, p.elem, false, g);
            store4(p.u_out, row, r0, p.cols, p.elem, false, u);
          }
        } else {
#pragma unroll
          for (int hb = 0; hb < 2; ++hb) {
            const int64_t r = r0 + kHalfRows * hb;
            if (r >= p.cols) continue;
            store4(p.out[z], row, r, p.cols, p.out_type, p.accumulate,
                   scaled4(acc[ha][hb][i][j], st, p.wide_scale[0], r, p.cols));
          }
        }
      }
    }
}

template <int ELEM, bool WS, bool TS, bool GATED>
void launch_tiles(const Product& p, hipStream_t stream) {
  const int64_t per = GATED ? 128 : 256;
  const int64_t tiles = (p.cols + per - 1) / per * ((p.rows + 255) / 256) * p.batch;
  wide_kernel<ELEM, WS, TS, GATED><<<dim3(static_cast<unsigned>(tiles)), 512, 0, stream>>>(p);
}

template <int ELEM>
void launch_elem(const Product& p, hipStream_t stream) {
  if (p.gated) return launch_tiles<ELEM, false, false, true>(p, stream);
  if constexpr (ELEM == kElemI8) {
    launch_tiles<ELEM, false, false, false>(p, stream);
  } else if (p.tall_strided) {
    launch_tiles<ELEM, true, true, false>(p, stream);
  } else {
    launch_tiles<ELEM, true, false, false>(p, stream);
  }
}

}  // namespace

void launch_wide(const Product& p, hipStream_t stream) {
  if (p.elem == kElemF16) launch_elem<kElemF16>(p, stream);
  else if (p.elem == kElemBf16) launch_elem<kElemBf16>(p, stream);
  else launch_elem<kElemI8>(p, stream);
}

}  // namespace sdq
