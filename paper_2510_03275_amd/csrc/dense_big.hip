// The products of the dense operators on 256 x 256 tiles of four waves (dense.h), for
// operands whose rows start 16-byte aligned: the large products.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "dense_device.h"

namespace sdq {
namespace {

typedef __attribute__((address_space(3))) void* LdsPtr;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* LdsS4;

constexpr int kStepBytes = 128;                // of depth
constexpr int kOperand = 256 * kStepBytes;     // bytes of one operand's step in LDS
constexpr int kTallStages = 2, kWideStages = 3;
constexpr unsigned kOut = 0x80000000u;         // an offset past every buffer
constexpr int kRsrcWord3 = 0x00020000;
constexpr int kXcds = 8;

constexpr int wait_counts(int vm) { return (vm & 15) | ((vm >> 4) << 14) | (7 << 4); }   // and lgkmcnt(0)

// 16 bytes per lane from src + soff + off to LDS at lds + 16 lane; zeros from `end` bytes behind src on.
// Through the builtin the compiler waits for every copy in flight before it lets a transposed LDS
// read pass, since it cannot tell their places apart (depth-contiguous reads it lets pass).  UNSEEN,
// for the kernels with transposed reads: the same instruction as text, which has no output register
// to lose (five wait states in front of it: a scalar operand may have been written by a vector
// instruction); the counted waits of the main loop are what orders copies and reads in either form.
template <bool UNSEEN>
__device__ inline void copy_16(char* lds, const char* src, int end, unsigned off, int soff) {
  if constexpr (UNSEEN) {
    const uint64_t at = reinterpret_cast<uint64_t>(src);
    const i32x4 rs = {static_cast<int>(at), static_cast<int>(at >> 32) & 0xFFFF, end, kRsrcWord3};
    const unsigned to = static_cast<unsigned>(reinterpret_cast<uintptr_t>((LdsPtr)lds));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(off), "s"(rs),
                 "s"(soff)
                 : "memory");      // m0 has no other use in these kernels
  } else {
    const __amdgpu_buffer_rsrc_t rs =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(src), static_cast<short>(0), end, kRsrcWord3);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (LdsPtr)lds, 16, off, soff, 0, 0);
  }
}

// The copies of a workgroup's 256 rows of an operand, one step after the other: four per wave and
// step.  Depth-contiguous: the descriptors stay (of two halves for gate and up) and the step is the
// scalar offset.  Strided: the descriptor moves, and ends with the depth.  Scalars that are compared
// are 32 bits wide: no branch splits the loop.
template <int BYTES, bool STRIDED, bool HALVES>
struct Loader {
  static constexpr int kStep = kStepBytes / BYTES;
  const char* src[HALVES ? 2 : 1];
  int num[HALVES ? 2 : 1];   // depth-contiguous: bytes from src to the last row's end
  const char* second;        // the other segment
  int64_t step;              // strided: bytes of a step
  int soff;                  // depth-contiguous: bytes of the steps done
  int depth, left;           // of the segment: in bytes (depth-contiguous) or depths
  int row_bytes, skip;       // strided: of one depth, and in front of the rows
  unsigned off[4];           // the lane's source offsets
  int chunk;                 // its place in a step's 128 bytes (depth-contiguous)

  // Rows r0 .. of n rows, from step t on; steps per segment.
  __device__ inline void init(const void* first, const void* other, int64_t r0, int64_t n, int64_t ld, int64_t depth_,
                              int t, int steps, int wave, int lane) {
    const unsigned ld_bytes = static_cast<unsigned>(ld * BYTES);
    const int past = t < steps ? t : t - steps;
    const int64_t at = r0 * (STRIDED ? 1 : ld) * BYTES;
    const int valid = static_cast<int>(n) - static_cast<int>(r0);
    if (STRIDED) {
      // LDS: [half][64 depths][128 elements]: copy j of wave w holds depths 4 (w + 8 (j % 2)) .. + 3 of half j / 2
      depth = static_cast<int>(depth_);
      step = kStep * static_cast<int64_t>(ld_bytes);
      src[0] = static_cast<const char*>(t < steps ? first : other) + at + past * step;
      second = static_cast<const char*>(other) + at;
      row_bytes = static_cast<int>(ld_bytes);
      skip = static_cast<int>(r0) * BYTES;
      const int swz = ((lane / 16) << 1) | (wave / 2 % 2);
      const int r = (((lane % 16) / 2) ^ swz) * 16 + (lane % 2) * 8;
      for (int j = 0; j < 4; ++j) off[j] = (4 * wave + lane / 16 + 32 * (j % 2)) * ld_bytes + 2 * (r + 128 * (j / 2));
      left = depth - past * kStep;
      chunk = soff = 0;
    } else {
      // LDS: [256 rows][128 bytes]: copy j of wave w holds rows 8 (w + 8 j) .. + 7
      depth = static_cast<int>(depth_ * BYTES);
      src[0] = static_cast<const char*>(t < steps ? first : other) + at;
      second = static_cast<const char*>(other) + at;
      num[0] = min(valid, HALVES ? 128 : 256) * static_cast<int>(ld_bytes);
      if (HALVES) {
        src[HALVES] = second;
        num[HALVES] = num[0];
      }
      chunk = 16 * ((lane % 8) ^ (lane / 8));
      for (int j = 0; j < 4; ++j) off[j] = (8 * wave + lane / 8 + 64 * (HALVES ? j % 2 : j)) * ld_bytes + chunk;
      soff = past * kStepBytes;
      left = depth - soff;
      row_bytes = skip = 0;
    }
  }
  // The next step to LDS.  MASK: it may be a segment's last or (unless `read`) behind it: zeros past
  // the depth.  restart: the other segment begins.
  template <bool MASK, bool SEGMENTS, bool UNSEEN>
  __device__ inline void copy(char* lds, int wave, bool read, bool restart) {
    if (SEGMENTS) {
      src[0] = restart ? second : src[0];
      left = restart ? depth : left;
      soff = restart ? 0 : soff;
    }
    const int have = MASK && !read ? 0 : left;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int h = HALVES ? j / 2 : 0;
      // Strided: columns behind the operand's last belong to the next depth: they are read, and their
      // outputs not stored.
      const int end = STRIDED ? max(min(have, kStep) * row_bytes - skip, 0) : num[h];
      const unsigned o = MASK && !STRIDED && chunk >= have ? kOut : off[j];
      copy_16<UNSEEN>(lds + j * 8192 + wave * 1024, src[h], end, o, STRIDED ? 0 : soff);
    }
    if (STRIDED) src[0] += step;
    else soff += kStepBytes;
    left -= STRIDED ? kStep : kStepBytes;
  }
};

// The lane's places in an operand's step for a wave's 16 N rows from row0 on.
template <bool STRIDED, int N>
struct Frags {
  int at[STRIDED ? N : 2];
  __device__ inline void init(int row0, int lane) {
    const int g = lane / 16, i = lane % 16;
    if (STRIDED) {
      for (int n = 0; n < N; ++n) {
        const int granule = (row0 % 128 / 16 + n) ^ (((i / 4) << 1) | (g % 2));
        at[n] = row0 / 128 * (kOperand / 2) + (8 * g + i / 4) * 256 + granule * 32 + (i % 4) * 8;
      }
    } else {
      for (int s = 0; s < 2; ++s) at[s] = (row0 + i) * kStepBytes + (((4 * s + g) ^ (i % 8)) * 16);
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
      return *reinterpret_cast<const i32x4*>(lds + at[s] + n * 16 * kStepBytes);
    }
  }
};

template <int ELEM, bool WIDE_STRIDED, bool TALL_STRIDED, bool GATED>
__global__ __launch_bounds__(512, 2) void big_kernel(Product p, int splits) {
  using E = Elem<ELEM>;
  using Acc = typename E::Acc;
  constexpr int kB = E::kBytes, kStep = kStepBytes / kB;
  __shared__ __attribute__((aligned(1024))) char lds[(kTallStages + kWideStages) * kOperand];   // stages of tall, of wide
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int ww = wave % 4, wt = wave / 4;

  constexpr int kCols = GATED ? 128 : 256;
  const unsigned nw = static_cast<unsigned>((p.cols + kCols - 1) / kCols);
  const unsigned nt = static_cast<unsigned>((p.rows + 255) / 256);
  const unsigned total = gridDim.x, id = blockIdx.x;
  const unsigned xcd = id % kXcds, per = total / kXcds, rem = total % kXcds;
  unsigned tile = xcd * per + (xcd < rem ? xcd : rem) + id / kXcds;
  const int part = __builtin_amdgcn_readfirstlane(tile / (nw * nt));
  tile -= part * (nw * nt);
  const int z = splits > 1 ? 0 : part;
  const unsigned band = tile / (4 * nw), in_band = tile - band * (4 * nw);
  const unsigned band_rows = nt - 4 * band < 4 ? nt - 4 * band : 4;
  const unsigned tw = in_band / band_rows, tt = 4 * band + (in_band - tw * band_rows);
  const int64_t row0 = static_cast<int64_t>(__builtin_amdgcn_readfirstlane(tt)) * 256;
  const int64_t col0 = static_cast<int64_t>(__builtin_amdgcn_readfirstlane(tw)) * kCols;

  const int seg_steps = static_cast<int>((p.depth + kStep - 1) / kStep), steps = seg_steps * p.segments;
  const int each = steps / splits, more = steps % splits, at = splits > 1 ? part : 0;
  const int t0 = at * each + min(at, more), t1 = t0 + each + (at < more ? 1 : 0);

  constexpr bool kSegments = WIDE_STRIDED && !TALL_STRIDED;      // two in the gradient of the block's input only
  Loader<kB, TALL_STRIDED, false> la;
  Loader<kB, WIDE_STRIDED, GATED> lb;
  la.init(p.tall[p.batch > 1 ? z : 0], p.tall[1], row0, p.rows, p.ld_tall, p.depth, t0, seg_steps, wave, lane);
  lb.init(p.wide[0], p.wide[1], col0, p.cols, p.ld_wide, p.depth, t0, seg_steps, wave, lane);
  Frags<TALL_STRIDED, 8> fa;
  Frags<WIDE_STRIDED, 4> fb;
  fa.init(128 * wt, lane);
  fb.init(64 * ww, lane);

  // LDS offsets of the stages read and filled next.
  constexpr int kWide = kTallStages * kOperand, kEnd = kWide + kWideStages * kOperand;
  int get_a = 0, get_b = kWide, put_a = 0, put_b = kWide;
  auto next_a = [](int at) { return at + kOperand == kWide ? 0 : at + kOperand; };
  auto next_b = [](int at) { return at + kOperand == kEnd ? kWide : at + kOperand; };
  auto restart = [&](int t) { return kSegments && t == seg_steps && t0 < seg_steps; };
  auto copy_a = [&](int t, auto mask) {
    la.template copy<decltype(mask)::value, kSegments, WIDE_STRIDED>(lds + put_a, wave, t < t1, restart(t));
    put_a = next_a(put_a);
  };
  auto copy_b = [&](int t, auto mask) {
    lb.template copy<decltype(mask)::value, kSegments, WIDE_STRIDED>(lds + put_b, wave, t < t1, restart(t));
    put_b = next_b(put_b);
  };

  Acc acc[8][4] = {};        // [rows of tall / 16][rows of wide / 16]
  i32x4 a[2][8], b[2][4];    // [depth half][rows / 16]
  auto read = [&](int s) {
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      a[s][n] = fa.read(lds + get_a, n, s);
      if (n % 2) b[s][n / 2] = fb.read(lds + get_b, n / 2, s);
    }
  };
  auto multiply = [&](int s) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = E::mfma(b[s][j], a[s][i], acc[i][j]);
  };
  // What was read has arrived, and all copies but the newest of wide, of every wave.
  auto turn = [&](auto newer) {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(wait_counts(decltype(newer)::value));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };
  auto spread = [&](auto copies) {
    constexpr int kReads = (TALL_STRIDED ? 2 : 1) * 8 + (WIDE_STRIDED ? 2 : 1) * 4;
    constexpr int kCopies = decltype(copies)::value;
#pragma unroll
    for (int n = 0; n < kCopies; ++n) {
      __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    }
#pragma unroll
    for (int n = 0; n < kReads; ++n) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, kReads > 12 ? 1 : kCopies ? 1 : 2, 0);
    }
  };

  typedef std::integral_constant<int, 0> C0;
  typedef std::integral_constant<int, 4> C4;
  typedef std::integral_constant<int, 8> C8;
  typedef std::integral_constant<int, 12> C12;
  copy_a(t0, std::true_type());
  copy_b(t0, std::true_type());
  copy_a(t0 + 1, std::true_type());
  copy_b(t0 + 1, std::true_type());
  copy_b(t0 + 2, std::true_type());
  turn(C12());
  read(0);
  auto step = [&](int t, auto mask) {
    read(1);
    multiply(0);
    spread(C0());
    turn(C4());              // step t is in registers, step t + 1 in LDS
    copy_a(t + 2, mask);
    copy_b(t + 3, mask);
    get_a = next_a(get_a);
    get_b = next_b(get_b);
    read(0);
    multiply(1);
    spread(C8());
    __builtin_amdgcn_sched_barrier(0);
  };
  // Steps that no copy has to be masked for: all but a segment's last.
  const int whole = p.depth % kStep == 0 ? t1 : kSegments ? t0 : min(t1, seg_steps - 1);
  int t = t0;
  for (; t + 3 < whole; ++t) step(t, std::false_type());
  for (; t < t1; ++t) step(t, std::true_type());
  __builtin_amdgcn_s_waitcnt(0);      // the copies past the end land before the sums take their place
  __syncthreads();

  // Sums of half a tile, 64 rows of either half of tall: [128 rows][64 chunks of four columns], chunk
  // q of row r at q ^ (r % 16).
  Acc* sums = reinterpret_cast<Acc*>(lds);
  const int64_t ld_part = (p.cols + 3) / 4 * 4;
#pragma unroll
  for (int pass = 0; pass < 2; ++pass) {
    if (pass) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = 64 * wt + 16 * i + lane % 16, q = 16 * ww + 4 * j + lane / 16;
        sums[r * 64 + (q ^ (r % 16))] = acc[4 * pass + i][j];
      }
    __syncthreads();
    if (splits > 1) {
#pragma unroll 2
      for (int o = tid; o < 128 * 64; o += 512) {
        const int r = o / 64, q = o % 64;
        const int64_t row = row0 + 128 * (r / 64) + 64 * pass + r % 64, c = col0 + 4 * (GATED ? q % 32 : q);
        if (row >= p.rows || c >= p.cols) continue;
        Acc* dst = static_cast<Acc*>(p.ws) + (part * p.rows + row) * ((GATED ? 2 : 1) * ld_part / 4) +
                    (GATED ? q / 32 : 0) * (ld_part / 4) + c / 4;
        *dst = sums[r * 64 + (q ^ (r % 16))];
      }
      continue;
    }
    constexpr int kOuts = GATED ? 32 : 64;
#pragma unroll 2
    for (int o = tid; o < 128 * kOuts; o += 512) {
      const int r = o / kOuts, q = o % kOuts;
      const int64_t row = row0 + 128 * (r / 64) + 64 * pass + r % 64, c = col0 + 4 * q;
      if (row >= p.rows || c >= p.cols) continue;
      finish4<ELEM, GATED>(p, z, row, c, sums[r * 64 + (q ^ (r % 16))],
                           GATED ? sums[r * 64 + ((q + 32) ^ (r % 16))] : Acc{});
    }
  }
}

template <int ELEM, bool WS, bool TS, bool GATED>
void launch_tiles(const Product& p, int splits, hipStream_t stream) {
  const int64_t per = GATED ? 128 : 256;
  const int64_t tiles = (p.cols + per - 1) / per * ((p.rows + 255) / 256);
  big_kernel<ELEM, WS, TS, GATED><<<dim3(static_cast<unsigned>(tiles * p.batch * splits)), 512, 0, stream>>>(p, splits);
}

template <int ELEM>
void launch_elem(const Product& p, int splits, hipStream_t stream) {
  if (p.gated) return launch_tiles<ELEM, false, false, true>(p, splits, stream);
  if constexpr (ELEM == kElemI8) launch_tiles<ELEM, false, false, false>(p, splits, stream);
  else if (p.tall_strided) launch_tiles<ELEM, true, true, false>(p, splits, stream);
  else launch_tiles<ELEM, true, false, false>(p, splits, stream);
}

}  // namespace

void launch_big(const Product& p, int splits, hipStream_t stream) {
  if (p.elem == kElemF16) launch_elem<kElemF16>(p, splits, stream);
  else if (p.elem == kElemBf16) launch_elem<kElemBf16>(p, splits, stream);
  else launch_elem<kElemI8>(p, splits, stream);
}

}  // namespace sdq
