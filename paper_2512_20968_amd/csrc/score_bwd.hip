// Backward of the tile attention under a score rule (mesh_attn_score_bwd),
// gfx950.  Deterministic: every output element is owned by one thread, no atomics.
//
// With P = exp(x - LSE) over the keys that are seen and T' = 1 - tanh^2 of the cap
// (4 r (1 - r) with the r of cap_r()):  dV = P^T dO,  dS = P T' (dO V^T - D),
// D = <dO, O>,  dK = s dS^T Q,  dQ = s dS K.  (Under a wide cap small arguments of
// the tanh take its series, and T' is 1 - tanh^2 of that.)
//
// Two launches, and one more for each pass whose items are cut:
//  1. prep: D and LSE log2(e) of every (row, head); every row's range and
//     position; what each stage of 64 rows sees.
//  2. dK/dV: a workgroup per (128 keys, KV head), four waves of 32 keys; it walks
//     the stages of 64 query rows that see some of its keys for every query head
//     of the group.  K, V, dK and dV stay in registers, which leaves room for the
//     exponentials of four queries at a time.
//  3. dQ, in the same launch: a workgroup per (128 rows, head), four waves of 32
//     rows, as the forward.
// The scores are made in both passes: seven products for the five that the
// gradients need.
//
// Bound by the matrix and the vector unit together (8192 causal rows of 32/8 heads
// of 128, matrix unit busy 47 % of the time, vector unit 54 %): with a cap 2024 to
// 2150 us, 0.64 to 0.68 PFLOP/s of the five products, 0.90 to 0.95 of the seven,
// where a large product reaches 1.22; without 1747 to 1790 us.  Documents in 4096
// rows 159 to 163 us; under the profiler prep takes 14 (a read of O and dO at the
// card's rate), the main kernel 142 to 151 and the sum of parts 13.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "internal.h"
#include "score_tile.h"

namespace mesh_attn {
namespace {

using namespace dev;

constexpr int NT = 256;

// Stages of a part of a dK/dV item, so that the keys of a long document do not take
// much longer than the rest.
constexpr int kPartStages = 8;

// ---------------------------------------------------------------------------
// 1. prep
// ---------------------------------------------------------------------------

// The first workgroups make the rows' ranges, a stage of 64 rows per wave; the
// others D and the LSE, D / 8 lanes per (row, head).
template <int D>
__global__ __launch_bounds__(NT) void score_prep_kernel(ScoreBwdParams p,
                                                        int range_groups) {
  const ScoreTile& t = p.t;
  const int tid = threadIdx.x;
  if (static_cast<int>(blockIdx.x) < range_groups) {
    const int stage = blockIdx.x * (NT / 64) + (tid >> 6);
    if (stage * 64 >= p.rows_pad) return;
    const int my = stage * 64 + (tid & 63);
    // Rows behind the last one see nothing, and count in no stage's summary.
    const int row = min(my, t.rows_q - 1);
    const int pos = row_position(t, row);
    const Seen s = row_seen(t, row, pos);
    p.lo[my] = my < t.rows_q ? s.lo : 0;
    p.hi[my] = my < t.rows_q ? s.hi : 0;
    p.pos[my] = pos;
    ScoreStage g;
    g.pos = __builtin_amdgcn_readfirstlane(pos);
    const int rel = pos - g.pos;
    g.wide = wave_max(abs(rel)) >= 1 << 23;
    p.pos_rel[my] = g.wide ? __int_as_float(rel) : static_cast<float>(rel);
    const bool some = s.lo < s.hi;
    g.lo_min = wave_min(some ? s.lo : INT32_MAX);
    g.hi_max = wave_max(s.hi);
    g.lo_max = wave_max(s.lo);
    g.hi_min = wave_min(s.hi);
    if (stage * 64 + 64 > t.rows_q) g.hi_min = 0;  // padding is masked
    if ((tid & 63) == 0) p.stages[stage] = g;
    return;
  }
  constexpr int kLanes = D / 8;
  const uint32_t gid = (blockIdx.x - range_groups) * NT + tid;
  const uint32_t item32 = gid / kLanes;  // row * hq + head
  const int sub = static_cast<int>(gid % kLanes);
  const int64_t row = item32 / static_cast<uint32_t>(t.hq);
  const int h = static_cast<int>(item32 - row * t.hq);
  const int64_t item = item32;
  const bool valid = row < t.rows_q;
  float s = 0.f;
  if (valid) {
    const bf16x8 a = *reinterpret_cast<const bf16x8*>(p.o + item * D + sub * 8);
    const bf16x8 b =
        *reinterpret_cast<const bf16x8*>(p.d_o + item * D + sub * 8);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      s = fmaf(static_cast<float>(a[i]), static_cast<float>(b[i]), s);
  }
#pragma unroll
  for (int o = kLanes / 2; o > 0; o /= 2) s += __shfl_xor(s, o);
  if (sub == 0 && row < p.rows_pad) {
    float lse = valid ? p.lse[int64_t{h} * t.rows_q + row] : -INFINITY;
    const int64_t at = int64_t{h} * p.rows_pad + row;
    // A D that is not finite makes the probabilities NaN instead, which hidden
    // pairs do not have.  (One that dO V^T could take to infinity counts as such;
    // rows without keys need none.)
    if (!(fabsf(s) < 0x1.cp127f) || lse == -INFINITY) {
      s = 0.f;
      if (lse != -INFINITY) lse = NAN;
    }
    p.delta[at] = -s;
    // Without the cap's constant part (see probability()).
    const float part = t.cap > kWideCap ? 0.f : t.cap;
    p.lse2[at] =
        lse == -INFINITY ? INFINITY : fmaf(lse, kLog2E, -part * kLog2E);
  }
}

// What the scores are put through: nothing, a cap, a wide one.
constexpr int kNoCap = 0, kCap = 1, kFineCap = 2;

// Scores x -> probability and, in *g, its product with the cap's derivative: a
// quarter of 4 r (1 - r), or 1 - tanh^2 of a wide one.  lse2: LSE less a cap that
// is not wide; far: |i - j|.
template <int CAP, bool BIAS>
__device__ __forceinline__ float probability(const Cap& cap, float scale_log2,
                                             float slope, float x, float far,
                                             float lse2, float* g) {
  float y, d = 1.f;
  if (CAP == kCap) {
    const float r = cap_r(cap, x);
    y = fmaf(-cap.two, r, -lse2);
    d = fmaf(-r, r, r);
  } else if (CAP == kFineCap) {
    const float u = x * cap.unit;
    const float h =
        fabsf(u) < kSeries ? tanh_series(u) : fmaf(-2.f, cap_r(cap, x), 1.f);
    y = fmaf(cap.one, h, -lse2);
    d = fmaf(-h, h, 1.f);
  } else {
    y = fmaf(x, scale_log2, -lse2);
  }
  if (BIAS) y = fmaf(-slope, far, y);
  const float e = exp2_fast(y);
  *g = CAP ? e * d : e;
  return e;
}

// The factor of dQ and dK that the sums lack.
template <int CAP>
__device__ __forceinline__ float grad_scale(const ScoreTile& t) {
  return CAP == kCap ? 4.f * t.scale : t.scale;
}

// Whether an operand holds large values or some that are not finite.
template <int N>
__device__ __forceinline__ bool holds_large(const bf16x8 (&f)[N]) {
  typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
  bool bad = false;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const u32x4v w = __builtin_bit_cast(u32x4v, f[i]);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      bad |= (w[j] & 0x7f80u) >= kLarge || (w[j] & 0x7f800000u) >= kLarge << 16;
  }
  return bad;
}

// ---------------------------------------------------------------------------
// 2. dK / dV
// ---------------------------------------------------------------------------
template <int D>
struct KvLayout {
  static constexpr int kTile = Staged<D>::kBytes;
  // Q, dO, then LSE, D, begin, end and position of 64 rows.
  static constexpr int kFloats = 2 * kTile;
  static constexpr int kStage = 2 * kTile + 5 * kScoreBlock * 4;
  static constexpr int kFlags = 2 * kStage;  // of the waves
  static constexpr int kLds = kFlags + 16;
};

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// Four values from LDS byte address a.
template <typename V4>
__device__ __forceinline__ V4 lds_four(uint32_t a) {
  typedef __attribute__((address_space(3))) const V4 T;
  return *(T*)a;
}

__device__ __forceinline__ void stage_words(const void* src, char* dst,
                                            int lane) {
  typedef __attribute__((address_space(3))) void lds_void;
  const rsrc_t r = make_rsrc(src, kScoreBlock * 4);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(dst), 4, lane * 4, 0,
                                           0, 0);
}

template <int D, int CAP, bool BIAS, bool OUT_F32>
__device__ __forceinline__ void dkdv_item(const ScoreBwdParams& p, char* smem,
                                          int id) {
  using L = KvLayout<D>;
  using T = Staged<D>;
  constexpr int kRow = T::kRowBytes;
  // P T' enters dS in float32, so that dS is rounded once.  At head dim 64 dO V^T is
  // held beside the scores.  At 128 that spills 31 to 89 registers: P goes into dV
  // first there, and P T' waits for dO V^T in the scores' registers (8192 causal
  // rows 2080 us, as with P T' in bf16, which left dK off by 0.0029 of its norm
  // instead of 0.0025).
  constexpr bool kBoth = D == 64;
  int* s_flags = reinterpret_cast<int*>(smem + KvLayout<D>::kFlags);
  const ScoreTile& t = p.t;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  const int hk = id % t.hkv;
  id /= t.hkv;
  // First parts first.  (With the parts of a block side by side, four of which one
  // has work, the items that have some all went to the same quarter of the compute
  // units: 842 us instead of 570.)
  const int part = id / t.kv_blocks128;
  int blk = id - part * t.kv_blocks128;
  Segment g;
  for (int s = 0; s < t.nseg; ++s) {
    g = segment(t, s);
    const int n = (g.len + kScoreRows - 1) / kScoreRows;
    if (blk < n) break;
    blk -= n;
  }
  // Keys behind the segment's last one repeat it, are seen by no row and not
  // stored.
  const int key0 = blk * kScoreRows, my_key = key0 + wave * 32 + li;
  const bool valid = my_key < g.len;
  const int key = min(my_key, g.len - 1);
  const int kpos = valid ? g.pos + key * t.step : INT32_MAX;
  const int wg_first = g.pos + key0 * t.step;
  const int wg_last =
      g.pos + (min(key0 + kScoreRows, g.len) - 1) * t.step;
  const int wave_first = __builtin_amdgcn_readfirstlane(
      g.pos + min(key0 + wave * 32, g.len - 1) * t.step);
  const int wave_last = __builtin_amdgcn_readfirstlane(
      g.pos + (min(key0 + wave * 32 + 32, g.len) - 1) * t.step);
  const bool wave_whole = key0 + wave * 32 + 32 <= g.len;
  const bool wg_whole = key0 + kScoreRows <= g.len;

  bf16x8 kf[D / 16], vf[D / 16];
  {
    const int64_t r = int64_t{g.row} + key;
    const uint16_t* ks = t.k + r * t.k_stride + int64_t{hk} * D + lh * 8;
    const uint16_t* vs = t.v + r * t.v_stride + int64_t{hk} * D + lh * 8;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      kf[kk] = *reinterpret_cast<const bf16x8*>(ks + kk * 16);
      vf[kk] = *reinterpret_cast<const bf16x8*>(vs + kk * 16);
    }
  }
  f32x16 acc_v[D / 32], acc_k[D / 32];
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    zero(acc_v[c]);
    zero(acc_k[c]);
  }
  const Cap cap = cap_of(t);

  // The stages that see some of the keys, 64 of them looked at at a time, for each
  // head of the group.
  const int stages = p.rows_pad / kScoreBlock;
  auto look = [&](int s0) {  // bits of the stages s0 ..
    const int s = s0 + lane;
    bool yes = false;
    if (s < stages) {
      const ScoreStage st = p.stages[s];
      yes = st.lo_min <= wg_last && st.hi_max > wg_first &&
            st.lo_min < st.hi_max;
    }
    return __builtin_amdgcn_ballot_w64(yes);
  };
  // This part's share of them.
  int skip = 0, take = INT32_MAX, parts = 1;
  if (p.kv_splits > 1) {
    int n = 0;
    for (int s0 = 0; s0 < stages; s0 += 64) n += __builtin_popcountll(look(s0));
    n *= t.group;
    parts = min(max((n + p.part_stages - 1) / p.part_stages, 1), p.kv_splits);
    if (part >= parts) return;
    skip = static_cast<int>(int64_t{n} * part / parts);
    take = static_cast<int>(int64_t{n} * (part + 1) / parts) - skip;
    if (part == 0 && tid < kScoreRows && key0 + tid < g.len)
      p.kv_parts[(int64_t{g.row} + key0 + tid) * t.hkv + hk] = parts;
  }
  int gh_next = 0, s_next = -64;  // where `bits` are from
  uint64_t bits = 0;
  // The next stage as group head * stages + stage; -1: there is none.
  auto next_stage = [&]() {
    if (take == 0) return -1;
    while (bits == 0) {
      s_next += 64;
      if (s_next >= stages) {
        s_next = 0;
        if (++gh_next >= t.group) return -1;
      }
      bits = look(s_next);
      const int n = __builtin_popcountll(bits);
      if (n <= skip) {
        skip -= n;
        bits = 0;
      }
    }
    for (; skip > 0; --skip) bits &= bits - 1;
    const int i = __builtin_ctzll(bits);
    bits &= bits - 1;
    --take;
    return gh_next * stages + s_next + i;
  };
  auto load = [&](int at, int buf) {
    // Not known to be the same from call to call: the loads' offsets are made
    // here instead of being held in registers through the loop.
    int lane = tid & 63;
    asm volatile("" : "+v"(lane));
    char* dst = smem + buf * L::kStage;
    const int gh = at / stages, s = at - gh * stages;
    const int h = hk * t.group + gh;
    const int64_t row = int64_t{s} * kScoreBlock;
    stage_rows<D>(t.q, t.q_stride, row, t.rows_q, h, dst, wave, lane);
    stage_rows<D>(p.d_o, int64_t{t.hq} * D, row, t.rows_q, h, dst + L::kTile,
                  wave, lane);
    char* f = dst + L::kFloats;
    const int64_t hr = int64_t{h} * p.rows_pad + row;
    if (wave == 0) stage_words(p.lse2 + hr, f, lane);
    if (wave == 1) stage_words(p.delta + hr, f + 256, lane);
    if (wave == 2) stage_words(p.lo + row, f + 512, lane);
    if (wave == 3) stage_words(p.hi + row, f + 768, lane);
    if (BIAS && wave == 0) stage_words(p.pos_rel + row, f + 1024, lane);
  };

  int cur = __builtin_amdgcn_readfirstlane(next_stage());
  if (cur >= 0) {
    load(cur, 0);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      wait_for(kf[kk]);
      wait_for(vf[kk]);
    }
    wait_vmem();
    __syncthreads();
    int buf = 0;
    const bool keys_large = __any(holds_large(kf) || holds_large(vf));
    // Operand addresses with the stage's base in them.
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)smem;
    uint32_t ra = lds0 + T::row_read(lane);
    uint32_t t0 = lds0 + T::tr_read(lane, 0);
    uint32_t t1 = lds0 + T::tr_read(lane, 1);
    uint32_t fa = lds0 + L::kFloats + lh * 32;
    for (;;) {
      const int nxt = __builtin_amdgcn_readfirstlane(next_stage());
      if (nxt >= 0) load(nxt, buf ^ 1);
      const int gh = cur / stages;
      const ScoreStage st = load_const(p.stages, cur - gh * stages);
      const float slope =
          BIAS ? load_const(t.slopes, hk * t.group + gh) * kLog2E : 0.f;
      // 0 times an infinity or a NaN of a row that does not see the key is NaN:
      // in stages that some of the workgroup's pairs are hidden in, rows that
      // hold one give NaN to the keys that they see, and zeros to the products.
      // What products of large values overflow to is taken out the same way.
      uint64_t bad = 0;
      bool large = false;
      if (__builtin_expect(
              !wg_whole || st.lo_max > wg_first || st.hi_min <= wg_last, 0)) {
        char* at = smem + buf * L::kStage;
        if (__builtin_expect(tiles_reach<D, 2, kLarge>(at, tid, s_flags), 0)) {
          large = true;
          bad = rows_not_finite<D>(at, lane) |
                rows_not_finite<D>(at + L::kTile, lane);
          lds_barrier();  // every wave has looked
          clear_not_finite<D>(at, tid);
          clear_not_finite<D>(at + L::kTile, tid);
          lds_barrier();
        }
      }
      const bool touched = st.lo_min <= wave_last && st.hi_max > wave_first;
      if (touched) {
        const bool full = wave_whole && st.lo_max <= wave_first &&
                          st.hi_min > wave_last;
        const bool fix = large || (!full && keys_large);
        const float kpos_rel =
            BIAS && !st.wide ? static_cast<float>(kpos - st.pos) : 0.f;
#pragma unroll
        for (int qt = 0; qt < 2; ++qt) {
          auto product = [&](const bf16x8 (&f)[D / 16], int tile, f32x16 z) {
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
              z = mfma32(lds_row((ra ^ (32 * kk)) + tile + qt * 32 * kRow),
                         f[kk], z);
            pipeline_reads<D / 16, 1, 3>();
            return z;
          };
          // dO V^T - D: the accumulators start with -D.
          auto d_probs = [&]() {
            f32x16 z;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const f32x4 dlt = lds_four<f32x4>(
                  fa + 256 + 4 * (qt * 32 + (i >> 1) * 16 + (i & 1) * 4));
#pragma unroll
              for (int e = 0; e < 4; ++e) z[i * 4 + e] = dlt[e];
            }
            return product(vf, L::kTile, z);
          };
          f32x16 x, y;
          if (kBoth) y = d_probs();
          zero(x);
          x = product(kf, 0, x);
          // Four queries at a time: more would not fit the registers.
          bf16x4 p4[4], d4[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t at = fa + 4 * (qt * 32 + (i >> 1) * 16 + (i & 1) * 4);
            f32x4 lse = lds_four<f32x4>(at);
            if (__builtin_expect(!full, 0)) {
              const i32x4 lo = lds_four<i32x4>(at + 512);
              const i32x4 hi = lds_four<i32x4>(at + 768);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (kpos < lo[e] || kpos >= hi[e]) lse[e] = INFINITY;
            }
            f32x4 e4, g4, pos;
            if (BIAS) {
              pos = lds_four<f32x4>(at + 1024);
              if (__builtin_expect(st.wide, 0)) {
                // In 32 bits: what wraps is not seen.
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  pos[e] = static_cast<float>(static_cast<int>(
                      __float_as_uint(pos[e]) -
                      static_cast<uint32_t>(kpos - st.pos)));
              }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float far = BIAS ? fabsf(pos[e] - kpos_rel) : 0.f;
              float g1;
              e4[e] = probability<CAP, BIAS>(cap, t.scale_log2, slope,
                                             x[i * 4 + e], far, lse[e], &g1);
              g4[e] = kBoth ? g1 * y[i * 4 + e] : g1;
            }
            if (__builtin_expect(fix, 0)) {
              const uint32_t b4 = static_cast<uint32_t>(
                  bad >> (qt * 32 + (i >> 1) * 16 + 8 * lh + (i & 1) * 4));
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float nan = (b4 >> e) & 1 ? NAN : 0.f;
                const bool hidden = lse[e] == INFINITY;
                e4[e] = hidden ? 0.f : e4[e] + nan;
                g4[e] = hidden ? 0.f : g4[e] + nan;
              }
            }
            p4[i] = __builtin_convertvector(e4, bf16x4);
            if (kBoth) {
              d4[i] = __builtin_convertvector(g4, bf16x4);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) x[i * 4 + e] = g4[e];
              __builtin_amdgcn_sched_barrier(0);
            }
          }
          auto joined = [](const bf16x4 (&f)[4], int hh) {
            return __builtin_shufflevector(f[2 * hh], f[2 * hh + 1], 0, 1, 2, 3,
                                           4, 5, 6, 7);
          };
          auto add = [&](int c, int hh, const bf16x4 (&f)[4], int tile,
                         f32x16& acc) {
            acc = mfma32(joined(f, hh),
                         lds_tr(t0 ^ (64 * c), t1 ^ (64 * c),
                                tile + (2 * qt + hh) * 16 * kRow),
                         acc);
          };
          if (!kBoth) {
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
#pragma unroll
              for (int hh = 0; hh < 2; ++hh)
                add(c, hh, p4, L::kTile, acc_v[c]);
            pipeline_reads<D / 16, 2, 2>();
            y = d_probs();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              f32x4 g4;
#pragma unroll
              for (int e = 0; e < 4; ++e) g4[e] = x[i * 4 + e] * y[i * 4 + e];
              // A hidden pair's product with dO V^T is 0, whatever that is.
              if (__builtin_expect(fix, 0)) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (x[i * 4 + e] == 0.f) g4[e] = 0.f;
              }
              d4[i] = __builtin_convertvector(g4, bf16x4);
            }
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
#pragma unroll
              for (int hh = 0; hh < 2; ++hh) add(c, hh, d4, 0, acc_k[c]);
            pipeline_reads<D / 16, 2, 2>();
          } else {
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
#pragma unroll
              for (int hh = 0; hh < 2; ++hh) {
                add(c, hh, p4, L::kTile, acc_v[c]);
                add(c, hh, d4, 0, acc_k[c]);
              }
            pipeline_reads<D / 8, 2, 2>();
          }
        }
      }
      if (nxt < 0) break;
      wait_vmem();
      lds_barrier();
      const int d = buf ? -L::kStage : L::kStage;
      ra += d;
      t0 += d;
      t1 += d;
      fa += d;
      buf ^= 1;
      cur = nxt;
    }
  }

  // Register i of chunk c: key 8 (i / 4) + 4 lh + i % 4 of the wave, dim 32 c + li.
  int last = tid & 63;  // made again, as in load()
  asm volatile("" : "+v"(last));
  const int li2 = last & 31, lh2 = last >> 5;
  const bool whole = parts == 1;
  const int64_t all_out = int64_t{t.rows_kv} * t.hkv * D;
  const float out_scale = grad_scale<CAP>(t);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int k = key0 + wave * 32 + 8 * (i >> 2) + 4 * lh2 + (i & 3);
    if (k >= g.len) continue;
    const int64_t at = ((int64_t{g.row} + k) * t.hkv + hk) * D + li2;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      const float dv = acc_v[c][i], dk = acc_k[c][i] * out_scale;
      if (!whole) {
        p.part_dv[part * all_out + at + 32 * c] = dv;
        p.part_dk[part * all_out + at + 32 * c] = dk;
      } else if (OUT_F32) {
        static_cast<float*>(p.dv)[at + 32 * c] = dv;
        static_cast<float*>(p.dk)[at + 32 * c] = dk;
      } else {
        static_cast<__bf16*>(p.dv)[at + 32 * c] = static_cast<__bf16>(dv);
        static_cast<__bf16*>(p.dk)[at + 32 * c] = static_cast<__bf16>(dk);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// 3. dQ
// ---------------------------------------------------------------------------
template <int D>
struct QLayout {
  static constexpr int kTile = Staged<D>::kBytes;
  static constexpr int kStage = 2 * kTile;
  static constexpr int kLds = 2 * kStage;
};

template <int D, int CAP, bool BIAS, bool OUT_F32>
__device__ __forceinline__ void dq_item(const ScoreBwdParams& p, char* smem,
                                        int id) {
  using L = QLayout<D>;
  using T = Staged<D>;
  constexpr int kRow = T::kRowBytes;
  int* s_flags = reinterpret_cast<int*>(smem + KvLayout<D>::kFlags);
  const ScoreTile& t = p.t;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qblocks = (t.rows_q + kScoreRows - 1) / kScoreRows;
  const int hk = id % t.hkv;
  id /= t.hkv;
  const int h = hk * t.group + id % t.group;
  id /= t.group;
  const int part = id % p.q_splits;
  const int qblk = qblocks - 1 - id / p.q_splits;

  const int my_row = qblk * kScoreRows + wave * 32 + li;
  const int row = min(my_row, t.rows_q - 1);
  const int qpos = p.pos[row];
  const Seen seen{p.lo[row], p.hi[row]};
  const int64_t hr = int64_t{h} * p.rows_pad + row;
  const float lse2 = p.lse2[hr], neg_delta = p.delta[hr];
  bf16x8 qf[D / 16], dof[D / 16];
  {
    const uint16_t* qs = t.q + row * t.q_stride + int64_t{h} * D + lh * 8;
    const uint16_t* ds = p.d_o + (int64_t{row} * t.hq + h) * D + lh * 8;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      qf[kk] = *reinterpret_cast<const bf16x8*>(qs + kk * 16);
      dof[kk] = *reinterpret_cast<const bf16x8*>(ds + kk * 16);
    }
  }
  f32x16 acc[D / 32];
#pragma unroll
  for (int c = 0; c < D / 32; ++c) zero(acc[c]);
  const Cap cap = cap_of(t);
  const float slope = BIAS ? t.slopes[h] * kLog2E : 0.f;
  const ScoreStage s0 = load_const(p.stages, 2 * qblk);
  const ScoreStage s1 =
      load_const(p.stages, min(2 * qblk + 1, p.rows_pad / kScoreBlock - 1));
  const int lo_min = min(s0.lo_min, s1.lo_min);
  const int hi_max = max(s0.hi_max, s1.hi_max);
  // (Rows behind the last one see nothing here: their stages count as masked.)
  const int lo_max = max(s0.lo_max, s1.lo_max);
  const int hi_min = min(s0.hi_min, s1.hi_min);
  KeyWalk w;
  w.start(t, lo_min < hi_max ? lo_min : 0, lo_min < hi_max ? hi_max : 0, part,
          p.q_splits);

  if (w.left > 0) {
    auto load = [&](int buf) {
      char* at = smem + buf * L::kStage;
      const int64_t r = w.g.row + int64_t{w.blk} * kScoreBlock;
      stage_rows<D>(t.k, t.k_stride, r, t.rows_kv, hk, at, wave, lane);
      stage_rows<D>(t.v, t.v_stride, r, t.rows_kv, hk, at + L::kTile, wave,
                    lane);
    };
    int a, b, all_a, all_b, some_a, some_b;
    auto enter_segment = [&]() {
      a = rows_below(seen.lo, w.g.pos, w.g.len, t.step);
      b = rows_below(seen.hi, w.g.pos, w.g.len, t.step);
      if (a >= b) a = b = 0;
      all_a = wave_max(a);
      all_b = wave_min(b);
      some_a = wave_min(a < b ? a : INT32_MAX);
      some_b = wave_max(b);
    };
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)smem;
    uint32_t ra = lds0 + T::row_read(lane);
    uint32_t t0 = lds0 + T::tr_read(lane, 0);
    uint32_t t1 = lds0 + T::tr_read(lane, 1);
    // bad: keys that are not finite, cleared in LDS: the rows that see them get
    // NaN.
    auto compute = [&](int k0, int pos0, uint64_t bad) {
      const bool full = all_a <= k0 && k0 + kScoreBlock <= all_b;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        f32x16 x, y;
        zero(x);
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = neg_delta;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          x = mfma32(lds_row((ra ^ (32 * kk)) + kt * 32 * kRow), qf[kk], x);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          y = mfma32(lds_row((ra ^ (32 * kk)) + L::kTile + kt * 32 * kRow),
                     dof[kk], y);
        pipeline_reads<D / 8, 1, 3>();
        const float d0 = BIAS ? static_cast<float>(int64_t{qpos} - pos0 -
                                                   int64_t{t.step} *
                                                       (32 * kt + 8 * lh))
                              : 0.f;
        const float step = static_cast<float>(t.step);
        bf16x8 ds[2];
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          f32x8 g8;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float far =
                BIAS ? fabsf(fmaf(-step, static_cast<float>(16 * hh + e), d0))
                     : 0.f;
            float g1;
            probability<CAP, BIAS>(cap, t.scale_log2, slope, x[hh * 8 + e], far,
                                   lse2, &g1);
            g8[e] = g1 * y[hh * 8 + e];
          }
          if (!full || bad != 0) {
            const int j0 = k0 + 32 * kt + 16 * hh + 8 * lh;
            const uint32_t b8 = static_cast<uint32_t>(
                bad >> (32 * kt + 16 * hh + 8 * lh)) & 255u;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const bool sees = a <= j0 + e && j0 + e < b;
              const float nan = (b8 >> e) & 1 ? NAN : 0.f;
              g8[e] = sees ? g8[e] + nan : 0.f;
            }
          }
          ds[hh] = __builtin_convertvector(g8, bf16x8);
        }
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
            const bf16x8 k = lds_tr(t0 ^ (64 * c), t1 ^ (64 * c),
                                    (2 * kt + hh) * 16 * kRow);
            acc[c] = mfma32(k, ds[hh], acc[c]);
          }
        pipeline_reads<D / 16, 2, 2>();
      }
    };
    load(0);
    enter_segment();
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      wait_for(qf[kk]);
      wait_for(dof[kk]);
    }
    wait_vmem();
    __syncthreads();
    int buf = 0;
    for (;;) {
      const int k0 = w.blk * kScoreBlock;
      const int pos0 = w.g.pos + k0 * t.step;
      const bool all_see =
          lo_max <= pos0 && pos0 + int64_t{t.step} * (kScoreBlock - 1) < hi_min &&
          k0 + kScoreBlock <= w.g.len;
      const bool more = w.left > 1;
      const bool changed = more && w.next(t);
      if (more) load(buf ^ 1);
      // 0 times an infinity or a NaN of a hidden key is NaN.
      uint64_t bad = 0;
      if (!all_see) {
        char* at = smem + buf * L::kStage;
        if (__builtin_expect(tiles_reach<D, 1, kNotFinite>(at, tid, s_flags),
                             0)) {
          bad = rows_not_finite<D>(at, lane);
          lds_barrier();  // every wave has looked
          clear_not_finite<D>(at, tid);
          lds_barrier();
        }
      }
      if (some_a < k0 + kScoreBlock && k0 < some_b) compute(k0, pos0, bad);
      if (!more) break;
      if (changed) enter_segment();
      wait_vmem();
      lds_barrier();
      const int step = buf ? -L::kStage : L::kStage;
      ra += step;
      t0 += step;
      t1 += step;
      buf ^= 1;
    }
  }
  if (my_row >= t.rows_q) return;
  const bool whole = p.q_splits == 1;
  const int64_t o0 = (int64_t{my_row} * t.hq + h) * D;
  const int64_t all = int64_t{t.rows_q} * t.hq * D;
  const float out_scale = grad_scale<CAP>(t);
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int dim = c * 32 + g * 8 + lh * 4;
      f32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = acc[c][4 * g + e] * out_scale;
      if (!whole) {
        *reinterpret_cast<f32x4*>(p.part_dq + part * all + o0 + dim) = x;
      } else if (OUT_F32) {
        *reinterpret_cast<f32x4*>(static_cast<float*>(p.dq) + o0 + dim) = x;
      } else {
        bf16x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = static_cast<__bf16>(x[e]);
        *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p.dq) + o0 + dim) = y;
      }
    }
}

// Both passes in one launch: the dK/dV items first, the longest of a causal tile
// at their front, and dQ items wherever one of them ends.  (A wide cap's tanh and a
// bias beside each other take 179 registers at head dim 64: two workgroups.)
template <int D, int CAP, bool BIAS, bool OUT_F32>
__global__ __launch_bounds__(NT, D == 128 || CAP == kFineCap ? 2 : 3)
void score_bwd_kernel(ScoreBwdParams p) {
  extern __shared__ __align__(16) char smem[];
  const int id = blockIdx.x;
  if (id < p.kv_items)
    dkdv_item<D, CAP, BIAS, OUT_F32>(p, smem, id);
  else
    dq_item<D, CAP, BIAS, OUT_F32>(p, smem, id - p.kv_items);
}

// ---------------------------------------------------------------------------
// Sums of partial gradients, four elements a thread, in the parts' order.
// ---------------------------------------------------------------------------
struct SumParams {
  const float* src[2];
  void* dst[2];
  int64_t n;  // elements of one, a multiple of 4
  int32_t parts;
  // Parts of every `d` elements, or null: `parts` of all.  One part: the result is
  // there.
  const int32_t* counts;
  int32_t d;
};

template <bool OUT_F32>
__global__ __launch_bounds__(NT) void score_sum_kernel(SumParams p) {
  const float* src = p.src[blockIdx.y];
  void* dst = p.dst[blockIdx.y];
  const int64_t stride = int64_t{gridDim.x} * NT * 4;
  for (int64_t i = (int64_t{blockIdx.x} * NT + threadIdx.x) * 4; i < p.n;
       i += stride) {
    // (At most `parts`, whatever is read.)
    const int parts =
        p.counts ? min(p.counts[static_cast<uint64_t>(i) / uint32_t(p.d)],
                       p.parts)
                 : p.parts;
    if (parts <= 1) continue;
    f32x4 s = *reinterpret_cast<const f32x4*>(src + i);
#pragma unroll 4
    for (int k = 1; k < parts; ++k) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(src + k * p.n + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += x[e];
    }
    if (OUT_F32) {
      *reinterpret_cast<f32x4*>(static_cast<float*>(dst) + i) = s;
    } else {
      bf16x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = static_cast<__bf16>(s[e]);
      *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(dst) + i) = y;
    }
  }
}

hipError_t launch_sum(const SumParams& p, int arrays, bool out_f32,
                      hipStream_t stream) {
  const int64_t need = (p.n / 4 + NT - 1) / NT;
  const dim3 grid(static_cast<unsigned>(need < 8192 ? need : 8192),
                  static_cast<unsigned>(arrays));
  if (out_f32)
    hipLaunchKernelGGL(score_sum_kernel<true>, grid, dim3(NT), 0, stream, p);
  else
    hipLaunchKernelGGL(score_sum_kernel<false>, grid, dim3(NT), 0, stream, p);
  return hipGetLastError();
}

template <int D, int CAP, bool BIAS, bool OUT_F32>
hipError_t launch(const ScoreBwdParams& p, hipStream_t stream) {
  constexpr auto kernel = score_bwd_kernel<D, CAP, BIAS, OUT_F32>;
  constexpr int lds = KvLayout<D>::kLds;
  static_assert(lds >= QLayout<D>::kLds, "one launch for both passes");
  hipError_t e = ensure_dynamic_lds<kernel>(lds);
  if (e != hipSuccess) return e;
  const ScoreTile& t = p.t;
  const int range_groups = (p.rows_pad / 64 + NT / 64 - 1) / (NT / 64);
  const int64_t lanes = int64_t{p.rows_pad} * t.hq * (D / 8);
  hipLaunchKernelGGL(
      score_prep_kernel<D>,
      dim3(static_cast<unsigned>(range_groups + (lanes + NT - 1) / NT)),
      dim3(NT), 0, stream, p, range_groups);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  ScoreBwdParams q = p;
  q.part_stages = kPartStages;
  q.kv_items = t.kv_blocks128 * t.hkv * p.kv_splits;
  const int64_t q_items =
      (int64_t{t.rows_q} + kScoreRows - 1) / kScoreRows * t.hq * p.q_splits;
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(q.kv_items + q_items)),
                     dim3(NT), lds, stream, q);
  e = hipGetLastError();
  if (e == hipSuccess && p.kv_splits > 1) {
    SumParams s{{p.part_dk, p.part_dv},
                {p.dk, p.dv},
                int64_t{t.rows_kv} * t.hkv * D,
                p.kv_splits,
                p.kv_parts,
                D};
    e = launch_sum(s, 2, OUT_F32, stream);
  }
  if (e == hipSuccess && p.q_splits > 1) {
    SumParams s{{p.part_dq, nullptr},
                {p.dq, nullptr},
                int64_t{t.rows_q} * t.hq * D,
                p.q_splits,
                nullptr,
                D};
    e = launch_sum(s, 1, OUT_F32, stream);
  }
  return e;
}

template <int D, bool OUT_F32>
hipError_t launch_d(const ScoreBwdParams& p, hipStream_t stream) {
  if (p.t.cap > kWideCap)
    return p.t.slopes ? launch<D, kFineCap, true, OUT_F32>(p, stream)
                      : launch<D, kFineCap, false, OUT_F32>(p, stream);
  if (p.t.cap > 0.f)
    return p.t.slopes ? launch<D, kCap, true, OUT_F32>(p, stream)
                      : launch<D, kCap, false, OUT_F32>(p, stream);
  return p.t.slopes ? launch<D, kNoCap, true, OUT_F32>(p, stream)
                    : launch<D, kNoCap, false, OUT_F32>(p, stream);
}

}  // namespace

// Most parts so that dK/dV has 512 items, two for each of 256 compute units, and
// dQ 128 beside them; of dK/dV's, a block of keys has as many as it has stages for.
// Microseconds for dK/dV whole / cut so / for 1024 items:
//   documents in 4096 rows of 32/8 heads of 128     204/178/188
//   4096 and 8192 causal rows of those      853/606/582, 2101/2103/2096
//   prefixes in 3001 rows of 12/4 heads of 64        164/ 55/ 55
//   1000 causal rows of 8 heads of 128                70/ 56/ 55
// and for parts of 16 stages 170, 607, 2097, 75, 74.
void score_bwd_splits(const ScoreTile& t, int* kv_splits, int* q_splits) {
  auto parts = [](int64_t items, int64_t blocks, int64_t target) {
    const int64_t want = (target + items - 1) / items, most = blocks / 4;
    const int64_t n = want < most ? want : most;
    return static_cast<int>(n < 1 ? 1 : n > 32 ? 32 : n);
  };
  const int64_t stages = (int64_t{t.rows_q} + 63) / 64;
  *kv_splits = parts(int64_t{t.kv_blocks128} * t.hkv, stages * t.group,
                     512);
  *q_splits = parts((int64_t{t.rows_q} + kScoreRows - 1) / kScoreRows * t.hq,
                    t.kv_blocks64, 128);
}

hipError_t launch_score_bwd(const ScoreBwdParams& p, bool out_f32,
                            hipStream_t stream) {
  if (out_f32)
    return p.t.head_dim == 128 ? launch_d<128, true>(p, stream)
                               : launch_d<64, true>(p, stream);
  return p.t.head_dim == 128 ? launch_d<128, false>(p, stream)
                             : launch_d<64, false>(p, stream);
}

}  // namespace mesh_attn
