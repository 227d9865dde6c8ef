// Device helpers of the attention under a score rule (gfx950, wave64), shared by
// its forward and backward kernels.  MFMA and LDS conventions as in
// tile_common.h: score tiles are made with their first operand's rows in the
// bit-2/3-swapped order, so that accumulator register i of lane half h is row
// acc_row(i, h) of a 32-row tile and eight registers are the k-contiguous operand
// of the next product.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "score.h"
#include "tile_common.h"

namespace mesh_attn {
namespace dev {

constexpr float kLog2E = 1.4426950408889634f;
constexpr float kLn2 = 0.69314718055994531f;

typedef __attribute__((address_space(3))) char lds_char;

// Rows of a staged tile, 16-byte chunks XORed by row, so that rows and transposed
// 4 x 16 blocks are both read without bank conflicts.
template <int D>
struct Staged {
  static constexpr int kRowBytes = 2 * D;
  static constexpr int kChunks = D / 8;
  static constexpr int kBytes = kScoreBlock * kRowBytes;
  __device__ static int swz(int r) {
    return D == 128 ? 4 * (r & 3) + ((r >> 2) & 3)
                    : 4 * ((r >> 1) & 1) + ((r >> 2) & 3);
  }
  // Byte offsets of a lane's operand reads: rows (row acc order of li, + 32 t;
  // chunk 2 kk + lh: ^ 32 kk), and the two halves of a transposed one (columns
  // 32 c ..: ^ 64 c; rows 16 s ..: + 16 s rows).
  __device__ static int row_read(int lane) {
    const int r = mfma_row_perm(lane & 31);
    return r * kRowBytes + (((lane >> 5) ^ swz(r)) * 16);
  }
  __device__ static int tr_read(int lane, int half) {
    const int g16 = lane >> 4, s16 = lane & 15;
    const int c16 = 2 * (g16 & 1) + ((s16 & 3) >> 1);
    const int r = 8 * (g16 >> 1) + (s16 >> 2) + 4 * half;
    return r * kRowBytes + ((c16 ^ swz(r)) * 16) + 8 * (s16 & 1);
  }
};

// Rows row0 .. row0 + 63 of a head into a staged tile, by four waves; rows from
// `rows` on are zeros (the buffer's range ends there).  The whole offset is in the
// lane's register, which the range check covers.
template <int D>
__device__ __forceinline__ void stage_rows(const uint16_t* base, int64_t stride,
                                           int64_t row0, int64_t rows, int head,
                                           char* tile, int wave, int lane) {
  using T = Staged<D>;
  constexpr int kPer = 64 / T::kChunks;  // rows of a load
  const uint32_t row_bytes = static_cast<uint32_t>(stride * 2);
  const int64_t left = rows - row0;
  const uint32_t n = left < kScoreBlock ? static_cast<uint32_t>(left)
                                        : uint32_t{kScoreBlock};
  const rsrc_t r = make_rsrc(base + row0 * stride + int64_t{head} * D,
                             (n - 1) * row_bytes + 2 * D);
#pragma unroll
  for (int j = 0; j < 16 / kPer; ++j) {
    const int tr = wave * 16 + j * kPer;
    const int row = tr + lane / T::kChunks;
    const uint32_t off =
        row * row_bytes + ((lane % T::kChunks) ^ T::swz(row)) * 16;
    buffer_load16_lds(r, tile + tr * T::kRowBytes, off, 0);
  }
}

__device__ __forceinline__ bf16x8 lds_row(uint32_t a) {
  typedef __attribute__((address_space(3))) const bf16x8 T;
  return *(T*)a;
}
__device__ __forceinline__ bf16x8 lds_tr(uint32_t a0, uint32_t a1, int imm) {
  typedef __attribute__((address_space(3))) s16x4 T;
  return join_bf16(__builtin_amdgcn_ds_read_tr16_b64_v4i16((T*)(a0 + imm)),
                   __builtin_amdgcn_ds_read_tr16_b64_v4i16((T*)(a1 + imm)));
}

// Order of a block of N groups of G MFMAs with R LDS operand reads each: the
// reads of AHEAD groups in flight ahead of the group that uses them.
template <int N, int R, int AHEAD, int G = 1>
__device__ __forceinline__ void pipeline_reads() {
  __builtin_amdgcn_sched_group_barrier(0x100, R * AHEAD, 0);
#pragma unroll
  for (int i = 0; i < N - AHEAD; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, G, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, G * AHEAD, 0);
}

// Exponent bits of bf16 values: of infinities and NaN, and of 2^59, below which
// the sums of 128 products stay below 2^125.
constexpr uint32_t kNotFinite = 0x7f80, kLarge = 0x5d00;

// Whether some of `tiles` staged tiles one after the other hold a value with the
// exponent `kFrom` or above: every wave looks at a quarter, the answers meet in
// s_flags.  For all waves of the workgroup together; between two calls lies another
// barrier.
template <int D, int tiles, uint32_t kFrom>
__device__ __forceinline__ bool tiles_reach(const char* tile, int tid,
                                            int* s_flags) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
  typedef int i32x4v __attribute__((ext_vector_type(4)));
  u16x2 top = {0, 0};
#pragma unroll
  for (int i = 0; i < tiles * Staged<D>::kBytes / (16 * kThreads); ++i) {
    const u32x4v w = *reinterpret_cast<const u32x4v*>(
        tile + (i * kThreads + tid) * 16);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      top = __builtin_elementwise_max(
          top, __builtin_bit_cast(u16x2, w[j] & 0x7f807f80u));
  }
  const bool any = __any(top[0] >= kFrom || top[1] >= kFrom);
  if ((tid & 63) == 0) s_flags[tid >> 6] = any;
  lds_barrier();
  const i32x4v f = *reinterpret_cast<const i32x4v*>(s_flags);
  return __builtin_amdgcn_readfirstlane(f[0] | f[1] | f[2] | f[3]) != 0;
}

// The operand with zeros for what is not finite.
__device__ __forceinline__ bf16x8 finite_or_zero(bf16x8 a) {
  typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
  u16x8 w = __builtin_bit_cast(u16x8, a);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if ((w[i] & 0x7f80) == 0x7f80) w[i] = 0;
  return __builtin_bit_cast(bf16x8, w);
}

// Rows of a staged tile that hold an infinity or a NaN, as bits.
template <int D>
__device__ __forceinline__ uint64_t rows_not_finite(const char* tile,
                                                    int lane) {
  bool bad = false;
#pragma unroll 1
  for (int i = 0; i < Staged<D>::kRowBytes / 4; ++i) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(
        tile + lane * Staged<D>::kRowBytes + 4 * i);
    bad |= (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
  }
  return __builtin_amdgcn_ballot_w64(bad);
}

// Zeros for what is not finite in a staged tile, by the whole workgroup.
template <int D>
__device__ __forceinline__ void clear_not_finite(char* tile, int tid) {
#pragma unroll 1
  for (int i = tid; i < Staged<D>::kBytes / 16; i += kThreads) {
    bf16x8* at = reinterpret_cast<bf16x8*>(tile + 16 * i);
    *at = finite_or_zero(*at);
  }
}

// Which stored positions a query row sees, [lo, hi); lo = hi = 0 for none.
struct Seen {
  int lo, hi;
};
__device__ __forceinline__ int row_position(const ScoreTile& t, int row) {
  // (The first partition's number comes with the other arguments; a table entry is
  // another round trip to memory.)
  if (t.rows_q == t.P)
    return t.striped ? row * t.n + t.q_idx[0] : t.q_idx[0] * t.P + row;
  const int e = row / t.P, r = row - e * t.P;
  const int part = load_const(t.q_idx, e);
  return t.striped ? r * t.n + part : part * t.P + r;
}
__device__ __forceinline__ Seen row_seen(const ScoreTile& t, int row, int pos) {
  Seen s;
  s.lo = t.key_begin ? max(t.key_begin[row], 0) : 0;
  s.hi = t.key_end ? min(t.key_end[row], t.total)
                   : t.causal ? pos + 1 : t.total;
  if (s.lo >= s.hi) s.lo = s.hi = 0;
  return s;
}

// Rows of a segment of `len` rows from position pos0 on that lie below x.
__device__ __forceinline__ int rows_below(int x, int pos0, int len, int step) {
  if (x <= pos0) return 0;
  const uint32_t y = static_cast<uint32_t>(x) - static_cast<uint32_t>(pos0);
  const uint32_t n =
      step == 1 ? y
                : (y + static_cast<uint32_t>(step) - 1) /
                      static_cast<uint32_t>(step);
  return n < static_cast<uint32_t>(len) ? static_cast<int>(n) : len;
}

// x of all lanes joined by op (idempotent: a lane without a source joins its own),
// in the vector unit: sums over 2, 4, 8 and 16 lanes of a row, then over the rows.
// (Twelve of these through LDS permutes were a third of a short call.)
template <typename Op>
__device__ __forceinline__ int wave_reduce(int x, Op op) {
  x = op(x, __builtin_amdgcn_update_dpp(x, x, 0x111, 0xf, 0xf, false));
  x = op(x, __builtin_amdgcn_update_dpp(x, x, 0x112, 0xf, 0xf, false));
  x = op(x, __builtin_amdgcn_update_dpp(x, x, 0x114, 0xf, 0xf, false));
  x = op(x, __builtin_amdgcn_update_dpp(x, x, 0x118, 0xf, 0xf, false));
  x = op(x, __builtin_amdgcn_update_dpp(x, x, 0x142, 0xa, 0xf, false));
  x = op(x, __builtin_amdgcn_update_dpp(x, x, 0x143, 0xc, 0xf, false));
  return __builtin_amdgcn_readlane(x, 63);
}
__device__ __forceinline__ int wave_min(int x) {
  return wave_reduce(x, [](int a, int b) { return a < b ? a : b; });
}
__device__ __forceinline__ int wave_max(int x) {
  return wave_reduce(x, [](int a, int b) { return a > b ? a : b; });
}

// A segment of the KV buffer.
struct Segment {
  int row, pos, len;
};
__device__ __forceinline__ Segment segment(const ScoreTile& t, int s) {
  if (t.nseg == 1) return {0, t.seg_pos[0], t.rows_kv};
  Segment g;
  g.row = load_const(t.seg_row, s);
  g.len = load_const(t.seg_row, s + 1) - g.row;
  g.pos = load_const(t.seg_pos, s);
  return g;
}

// Walk over the 64-key blocks of all segments that positions [lo, hi) touch, or
// over part `part` of `parts` of them, from the last to the first: a bias is then
// largest at the start, and the softmax's reference seldom moves.  (8192 causal rows
// with a bias, first to last / so: 12 heads of 64 196/188 us, 32/8 of 128 642/592,
// float32 O 1003/923.)  Uniform over the workgroup.
struct KeyWalk {
  int seg, blk, begin, left, lo, hi;
  Segment g;

  __device__ int range(const ScoreTile& t) {  // blocks of the segment
    g = segment(t, seg);
    const int a = rows_below(lo, g.pos, g.len, t.step);
    const int b = rows_below(hi, g.pos, g.len, t.step);
    begin = __builtin_amdgcn_readfirstlane(a / kScoreBlock);
    const int n = a < b ? (b + kScoreBlock - 1) / kScoreBlock - begin : 0;
    blk = begin + __builtin_amdgcn_readfirstlane(n) - 1;
    return blk + 1 - begin;
  }
  __device__ void start(const ScoreTile& t, int lo_, int hi_, int part,
                        int parts) {
    lo = lo_;
    hi = hi_;
    left = 0;
    int skip = 0;
    if (parts > 1 || t.nseg > 1) {
      int all = 0;
      for (seg = 0; seg < t.nseg; ++seg) all += range(t);
      skip = static_cast<int>(int64_t{all} * part / parts);
      left = static_cast<int>(int64_t{all} * (part + 1) / parts) - skip;
      if (left == 0) return;
    }
    for (seg = t.nseg - 1; seg >= 0; --seg) {
      const int n = range(t);
      if (t.nseg == 1 && parts == 1) left = n;
      if (n > skip) {
        blk -= skip;
        return;
      }
      skip -= n;
    }
  }
  // To the next block; true if the segment changed.  Not past the last one.
  __device__ bool next(const ScoreTile& t) {
    --left;
    if (--blk >= begin || left <= 0) return false;
    do {
      --seg;
    } while (range(t) == 0);
    return true;
  }
};

// Scores of a 32-row tile in log2 units before the bias, and the cap's
// derivative.  tanh(u) = 1 - 2 / (1 + e^(2u)): one exponential and one reciprocal,
// off by 2^-23 of the cap; infinite products give +-cap.
struct Cap {
  float in;    // product -> log2(e^(2u))
  float two;   // 2 cap log2(e)
  float one;   // cap log2(e)
  float unit;  // product -> u
};
__device__ __forceinline__ Cap cap_of(const ScoreTile& t) {
  Cap c;
  c.in = t.cap > 0.f ? 2.f * t.scale_log2 / t.cap : 0.f;
  c.one = t.cap * kLog2E;
  c.two = 2.f * c.one;
  c.unit = t.cap > 0.f ? t.scale / t.cap : 0.f;
  return c;
}
__device__ __forceinline__ float cap_r(const Cap& c, float x) {
  return __builtin_amdgcn_rcpf(1.f + exp2_fast(x * c.in));
}

// tanh(u) for |u| < kSeries, off by a few 2^-24 of itself (1 - 2 r is by 2^-23 of
// one): Taylor; the first term left out is below 2^-23.9 of the sum.
constexpr float kSeries = 0.4f;
__device__ __forceinline__ float tanh_series(float u) {
  const float z = u * u;
  float s = fmaf(z, -1382.f / 155925, 62.f / 2835);
  s = fmaf(s, z, -17.f / 315);
  s = fmaf(s, z, 2.f / 15);
  s = fmaf(s, z, -1.f / 3);
  return fmaf(s * z, u, u);
}

}  // namespace dev
}  // namespace mesh_attn
