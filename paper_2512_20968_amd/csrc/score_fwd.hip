// Tile attention under a score rule, forward (mesh_attn_score_fwd), gfx950.
//
// x_ij = cap tanh(s <q_i, k_j> / cap) - slope_h |p_i - p_j| over the keys with
// begin_i <= p_j < end_i; O_i = sum_j exp(x_ij - LSE_i) v_j.
//
// One workgroup computes 128 query rows of a head, four waves of 32 rows, in one
// pass over the 64-key blocks that some row of them sees (a walk over the KV
// buffer's segments between the rows' least begin and largest end, which only the
// device knows), with the running maximum and sum of the softmax.  A wave whose
// rows see all of a block evaluates no mask; one whose rows see none of it skips
// it.  S^T = K Q^T and O^T += V^T P^T on v_mfma_f32_32x32x16_bf16: every lane owns
// a query row, Q and O stay in registers, K and V stream from memory straight into
// LDS, a block ahead.
//
// Bound by the vector unit (16384 causal rows of 32/8 heads of 128, cap: 2375 to
// 2490 us, 0.88 to 0.93 PFLOP/s; vector unit busy 0.75 of the time, matrix unit
// 0.45): a cap costs an exponential, a reciprocal and two more instructions per
// score beside the softmax's own.  Rows of a wave, 32: a range, a position and a
// slope per row are held beside O and Q, and two workgroups share a compute unit so
// that one's products run beside the other's exponentials.  Documents packed into
// 8192 rows 155 to 160 us, 0.5 PFLOP/s, by an uneven load (items come from the last
// rows on, not longest first) and the round trips at an item's start; 77 rows 9 us,
// all round trips.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "internal.h"
#include "score_tile.h"

namespace mesh_attn {
namespace {

using namespace dev;

constexpr int NT = 256;

// The reference of a row's probabilities may lag behind its maximum by this much
// (log2 units): they stay below 2^8, and the sums are rescaled a few times per
// row instead of whenever its maximum grows.  The first block's maximum is taken as
// it is: what is rounded of a row's only key, or of one that outweighs the rest,
// is 1.  (A fixed reference, which a moderate cap allows, saves 3 % and adds a
// rounding of 2^-8 to such rows.)
constexpr float kLag = 8.f;

template <int D>
struct Layout {
  static constexpr int kTile = Staged<D>::kBytes;
  static constexpr int kStage = 2 * kTile;  // K, V
  static constexpr int kLds = 2 * kStage + 20 * 4;  // .. the waves' ranges, flags
};

// EXACT (float32 O): the probabilities enter the second product as a sum of three
// bf16 that hold all 24 bits; else rounded to bf16, 2^-8 of each, as O itself is.
// FINE (float32 O, and wide caps): the tanh of small arguments is a polynomial.
template <int D, bool CAP, bool BIAS, bool EXACT, bool FINE>
__global__ __launch_bounds__(NT, D == 128 ? 2 : 3)
void score_fwd_kernel(ScoreFwdParams p) {
  using L = Layout<D>;
  using T = Staged<D>;
  constexpr int kRow = T::kRowBytes;
  extern __shared__ __align__(16) char smem[];
  // (The dynamic LDS starts at 0: operand addresses are XORed.)
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  i32x4* s_range = reinterpret_cast<i32x4*>(smem + 2 * L::kStage);
  const ScoreTile& t = p.t;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // Workgroup i runs on XCD i % 8: KV heads fastest, so that with 8 of them each
  // is read through one L2; the last rows, which see the most keys of a causal
  // tile, first.
  const int qblocks = (t.rows_q + kScoreRows - 1) / kScoreRows;
  int id = blockIdx.x;
  const int hk = id % t.hkv;
  id /= t.hkv;
  const int h = hk * t.group + id % t.group;
  id /= t.group;
  const int part = id % p.splits;
  const int qblk = qblocks - 1 - id / p.splits;

  // Rows behind the last one repeat it and are not stored.
  const int my_row = qblk * kScoreRows + wave * 32 + li;
  const int row = min(my_row, t.rows_q - 1);
  const int qpos = row_position(t, row);
  const Seen seen = row_seen(t, row, qpos);
  {
    // Positions that some row sees, and those that all rows see.
    const i32x4 r = {wave_min(seen.lo < seen.hi ? seen.lo : INT32_MAX),
                     wave_max(seen.hi), wave_max(seen.lo), wave_min(seen.hi)};
    if (lane == 0) s_range[wave] = r;
  }
  bf16x8 qf[D / 16];
  {
    const uint16_t* src = t.q + row * t.q_stride + int64_t{h} * D + lh * 8;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
      qf[kk] = *reinterpret_cast<const bf16x8*>(src + kk * 16);
  }
  f32x16 oacc[D / 32];
#pragma unroll
  for (int c = 0; c < D / 32; ++c) zero(oacc[c]);
  float m = -INFINITY, l = 0.f;
  const Cap cap = cap_of(t);
  // What is kept of a score: its product (scaled in the exponent), the r of the
  // cap (x = one - two r, the least of which is the largest score), or, with a
  // bias or where the tanh is fine, x itself in log2 units.
  constexpr bool kAsR = CAP && !BIAS && !FINE;
  const float unit = kAsR ? -cap.two : CAP || BIAS ? 1.f : t.scale_log2;
  const float base = kAsR ? cap.one : 0.f;
  const float slope = BIAS ? t.slopes[h] * kLog2E : 0.f;
  const int pos_min = BIAS ? wave_min(qpos) : 0;
  const int pos_max = BIAS ? wave_max(qpos) : 0;
  // The distance to the row's nearest key: biases are taken relative to it, so
  // that those of far keys keep their digits.
  int off = 0;
  if (BIAS) {
    int64_t nearest = INT64_MAX;
    for (int s = 0; s < t.nseg; ++s) {
      const Segment g = segment(t, s);
      const int a = rows_below(seen.lo, g.pos, g.len, t.step);
      const int b = rows_below(seen.hi, g.pos, g.len, t.step);
      if (a >= b) continue;
      const int at = rows_below(qpos, g.pos, g.len, t.step);  // first >= qpos
      const int64_t r0 = g.pos + int64_t{min(max(at, a), b - 1)} * t.step;
      const int64_t r1 = g.pos + int64_t{min(max(at - 1, a), b - 1)} * t.step;
      const int64_t d0 = r0 > qpos ? r0 - qpos : qpos - r0;
      const int64_t d1 = r1 > qpos ? r1 - qpos : qpos - r1;
      nearest = min(nearest, min(d0, d1));
    }
    off = nearest == INT64_MAX ? 0 : static_cast<int>(nearest);
  }
  __syncthreads();
  i32x4 range = s_range[0];
#pragma unroll
  for (int i = 1; i < 4; ++i) {
    const i32x4 r = s_range[i];
    range[0] = min(range[0], r[0]);
    range[1] = max(range[1], r[1]);
    range[2] = max(range[2], r[2]);
    range[3] = min(range[3], r[3]);
  }
  const int lo_min = __builtin_amdgcn_readfirstlane(range[0]);
  const int hi_max = __builtin_amdgcn_readfirstlane(range[1]);
  const int lo_max = __builtin_amdgcn_readfirstlane(range[2]);
  const int hi_min = __builtin_amdgcn_readfirstlane(range[3]);
  KeyWalk w;
  w.start(t, lo_min < hi_max ? lo_min : 0, lo_min < hi_max ? hi_max : 0, part,
          p.splits);

  if (w.left > 0) {
    auto load = [&](int buf) {
      char* at = smem + buf * L::kStage;
      const int64_t r = w.g.row + int64_t{w.blk} * kScoreBlock;
      stage_rows<D>(t.k, t.k_stride, r, t.rows_kv, hk, at, wave, lane);
      stage_rows<D>(t.v, t.v_stride, r, t.rows_kv, hk, at + L::kTile, wave,
                    lane);
    };
    // The rows' keys [a, b) in the segment, and over the wave: those that all
    // see and those that some see.
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
    // Operand addresses with the stage's base in them.
    uint32_t kra = lds0 + T::row_read(lane);
    uint32_t vt0 = lds0 + T::tr_read(lane, 0);
    uint32_t vt1 = lds0 + T::tr_read(lane, 1);

    // Values of a block that some of the workgroup's rows do not see, and that
    // are not finite, go straight to the rows that see them; the products get
    // zeros (0 times an infinity or a NaN is NaN).
    auto take_not_finite = [&](int k0, char* vt) {
#pragma unroll 1
      for (int j = 0; j < kScoreBlock; ++j) {
        if (j < a - k0 || j >= b - k0) continue;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const bf16x4 v4 = *reinterpret_cast<const bf16x4*>(
                vt + j * kRow + (((4 * c + g) ^ T::swz(j)) * 16) + 8 * lh);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float v = static_cast<float>(v4[e]);
              oacc[c][4 * g + e] += v - v == 0.f ? 0.f : v;
            }
          }
      }
      lds_barrier();  // every wave has read it
      clear_not_finite<D>(vt, tid);
      lds_barrier();
    };

    // One block: its first key is k0 of the segment, at position pos0.
    auto compute = [&](int k0, int pos0) {
      f32x16 sc[2];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        zero(sc[kt]);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          sc[kt] = mfma32(lds_row((kra ^ (32 * kk)) + kt * 32 * kRow), qf[kk],
                          sc[kt]);
      }
      pipeline_reads<D / 8, 1, 3>();
      if (CAP) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float x = sc[kt][i];
            if (kAsR) {
              sc[kt][i] = cap_r(cap, x);
              continue;
            }
            float y = fmaf(-cap.two, cap_r(cap, x), cap.one);
            if (FINE) {
              const float u = x * cap.unit;
              y = fabsf(u) < kSeries ? tanh_series(u) * cap.one : y;
            }
            sc[kt][i] = y;
          }
      } else if (BIAS) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[kt][i] *= t.scale_log2;
      }
      if (BIAS) {
        // Positions of the block: pos0 + step (0 .. 63), in 64 bits.
        const int64_t last = pos0 + int64_t{t.step} * (kScoreBlock - 1);
        const float step = static_cast<float>(t.step);
        if (last <= pos_min || pos0 >= pos_max) {
          const bool before = last <= pos_min;
          const float sg = before ? -step : step;
          const int64_t far =
              before ? int64_t{qpos} - pos0 : int64_t{pos0} - qpos;
          const float d0 = fmaf(sg, 8.f * lh, static_cast<float>(far - off));
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              sc[kt][i] = fmaf(
                  -slope, fmaf(sg, static_cast<float>(32 * kt + acc_row(i, 0)),
                               d0),
                  sc[kt][i]);
        } else {
          // A row before or behind all of the block's keys is as far from the
          // nearest end as `beyond` says: the rest is small enough for a float
          // (the rows of a wave may be of partitions that lie far apart).
          const int64_t at = int64_t{qpos} - pos0, end = last - pos0;
          const int64_t inside = at < 0 ? 0 : at > end ? end : at;
          const int64_t beyond = at < 0 ? -at : at > end ? at - end : 0;
          const float d0 = static_cast<float>(inside) - step * (8.f * lh);
          const float offf = static_cast<float>(off - beyond);
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float d =
                  fmaf(-step, static_cast<float>(32 * kt + acc_row(i, 0)), d0);
              sc[kt][i] = fmaf(-slope, fabsf(d) - offf, sc[kt][i]);
            }
        }
      }
      const bool full = all_a <= k0 && k0 + kScoreBlock <= all_b;
      if (!full) {
        const int x = a - k0 - 8 * lh, y = b - k0 - 8 * lh;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int j = 32 * kt + acc_row(i, 0);
            if (j < x || j >= y) sc[kt][i] = kAsR ? INFINITY : -INFINITY;
          }
      }
      float top = sc[0][0];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          top = kAsR ? fminf(top, sc[kt][i]) : fmaxf(top, sc[kt][i]);
      const float mx = max_with_other_half(fmaf(top, unit, base));
      if (__builtin_amdgcn_ballot_w64(mx > m + kLag)) {
        const float mn = fmaxf(m, mx);
        // (Sums before the first score are 0, or what take_not_finite() put
        // there, which a factor of 0 must not meet.)
        const float alpha =
            m == -INFINITY ? 1.f : fmaxf(exp2_fast(m - mn), 0x1p-126f);
        l *= alpha;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) oacc[c][i] *= alpha;
        m = mn;
      }
      const float ref = base - (m == -INFINITY ? 0.f : m);
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          sc[kt][i] = exp2_fast(fmaf(sc[kt][i], unit, ref));
          sum[i & 1] += sc[kt][i];
        }
      l += sum[0] + sum[1];
      bf16x8 pb[EXACT ? 3 : 1][4];
#pragma unroll
      for (int ss = 0; ss < 4; ++ss) {
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = sc[ss >> 1][(ss & 1) * 8 + i];
        if constexpr (EXACT) {
          typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
#pragma unroll
          for (int n = 0; n < 3; ++n) {
            u32x4v wd;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t e0 = __float_as_uint(e[2 * i]);
              const uint32_t e1 = __float_as_uint(e[2 * i + 1]);
              wd[i] = __builtin_amdgcn_perm(e1, e0, 0x07060302u);
              e[2 * i] -= __uint_as_float(e0 & 0xffff0000u);
              e[2 * i + 1] -= __uint_as_float(e1 & 0xffff0000u);
            }
            pb[n][ss] = __builtin_bit_cast(bf16x8, wd);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) pb[0][ss][i] = static_cast<__bf16>(e[i]);
        }
      }
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int ss = 0; ss < 4; ++ss) {
          const bf16x8 v = lds_tr(vt0 ^ (64 * c), vt1 ^ (64 * c),
                                  L::kTile + ss * 16 * kRow);
#pragma unroll
          for (int n = 0; n < (EXACT ? 3 : 1); ++n)
            oacc[c] = mfma32(v, pb[n][ss], oacc[c]);
        }
      pipeline_reads<D / 8, 2, EXACT ? 2 : 3, EXACT ? 3 : 1>();
    };

    load(0);
    enter_segment();
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) wait_for(qf[kk]);
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
      if (!all_see) {
        char* vt = smem + buf * L::kStage + L::kTile;
        if (__builtin_expect(
                tiles_reach<D, 1, kNotFinite>(
                    vt, tid, reinterpret_cast<int*>(s_range + 4)),
                0))
          take_not_finite(k0, vt);
      }
      if (some_a < k0 + kScoreBlock && k0 < some_b) compute(k0, pos0);
      if (!more) break;
      if (changed) enter_segment();
      wait_vmem();
      lds_barrier();  // the next stage has landed; this one has been read
      const int step = buf ? -L::kStage : L::kStage;
      kra += step;
      vt0 += step;
      vt1 += step;
      buf ^= 1;
    }
  }

  // O = acc / l, LSE = (m + log2 l - slope off) ln 2; 0 and -inf without a key.
  const float lt = l + __shfl_xor(l, 32);
  const float inv = lt > 0.f ? 1.f / lt : lt;
  float lse = lt == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(lt);
  if (m == -INFINITY && lt != 0.f) lse = lt;  // NaN
  if (BIAS) lse -= slope * static_cast<float>(off);
  if (my_row >= t.rows_q) return;
  const bool whole = p.splits == 1;
  const int64_t at = int64_t{h} * t.rows_q + my_row;
  const int64_t all = int64_t{t.hq} * t.rows_q;
  if (lh == 0) {
    float* dst = whole ? p.lse : p.part_lse + part * all;
    dst[at] = lse * kLn2;
  }
  const int64_t o0 = (int64_t{my_row} * t.hq + h) * D;
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int dim = c * 32 + g * 8 + lh * 4;
      f32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = oacc[c][4 * g + e] * inv;
      if (!whole) {
        *reinterpret_cast<f32x4*>(p.part_o + part * all * D + o0 + dim) = x;
      } else if (EXACT) {
        *reinterpret_cast<f32x4*>(static_cast<float*>(p.o) + o0 + dim) = x;
      } else {
        bf16x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = static_cast<__bf16>(x[e]);
        *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(p.o) + o0 + dim) = y;
      }
    }
}

template <int D, bool CAP, bool BIAS, bool EXACT, bool FINE>
hipError_t launch(const ScoreFwdParams& p, hipStream_t stream) {
  constexpr auto kernel = score_fwd_kernel<D, CAP, BIAS, EXACT, FINE>;
  constexpr int lds = Layout<D>::kLds;
  const hipError_t e = ensure_dynamic_lds<kernel>(lds);
  if (e != hipSuccess) return e;
  const int64_t blocks =
      (int64_t{p.t.rows_q} + kScoreRows - 1) / kScoreRows * p.t.hq * p.splits;
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(NT), lds,
                     stream, p);
  return hipGetLastError();
}

template <int D, bool EXACT>
hipError_t launch_d(const ScoreFwdParams& p, hipStream_t stream) {
  if (p.t.cap > kWideCap)
    return p.t.slopes ? launch<D, true, true, EXACT, true>(p, stream)
                      : launch<D, true, false, EXACT, true>(p, stream);
  if (p.t.cap > 0.f)
    return p.t.slopes ? launch<D, true, true, EXACT, EXACT>(p, stream)
                      : launch<D, true, false, EXACT, EXACT>(p, stream);
  return p.t.slopes ? launch<D, false, true, EXACT, EXACT>(p, stream)
                    : launch<D, false, false, EXACT, EXACT>(p, stream);
}

}  // namespace

// As many parts as fill the places of the 256 compute units (two workgroups each
// at head dim 128, three at 64).  Microseconds for 1 / this / twice as many:
// 3002 rows over 6004 striped keys, 12 heads of 64, float32 O 90 / 66 / 70; the
// same causal, bf16 161 / 82 / 77; 2000 causal rows, 4/2 heads of 64 44 / 22 / 22;
// 4096 causal rows, 8 heads of 128 101 / 73 / 77; 500 rows over 8000 keys, 8 of
// 128 183 / 39 / 56; window of 1024 in 4096 rows, 16/8 of 128 57 / 57 / 79.
int score_fwd_splits(const ScoreTile& t) {
  const int64_t items =
      (int64_t{t.rows_q} + kScoreRows - 1) / kScoreRows * t.hq;
  const int64_t places = t.head_dim == 128 ? 512 : 768;
  const int64_t want = (places + items - 1) / items, most = t.kv_blocks64 / 4;
  const int64_t n = want < most ? want : most;
  return static_cast<int>(n < 1 ? 1 : n > 64 ? 64 : n);
}

hipError_t launch_score_fwd(const ScoreFwdParams& p, bool out_f32,
                            hipStream_t stream) {
  hipError_t e;
  if (p.t.head_dim == 128)
    e = out_f32 ? launch_d<128, true>(p, stream)
                : launch_d<128, false>(p, stream);
  else
    e = out_f32 ? launch_d<64, true>(p, stream)
                : launch_d<64, false>(p, stream);
  if (e != hipSuccess || p.splits == 1) return e;
  MergeParams m;
  m.o_parts = p.part_o;
  m.lse_parts = p.part_lse;
  m.o_out = p.o;
  m.lse_out = p.lse;
  m.rows = p.t.rows_q;
  m.k_parts = p.splits;
  m.heads = p.t.hq;
  m.head_dim = p.t.head_dim;
  return launch_lse_merge(m, true, out_f32, stream);
}

}  // namespace mesh_attn
