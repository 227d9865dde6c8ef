// Attention of new query rows over the 4-bit paged cache (mesh_attn_cache_fwd).
//
// Mathematics: S^T = K Q^T, one pass over the keys with the running maximum and
// sum of the softmax, O^T += V^T P^T, all on v_mfma_f32_16x16x32_bf16.
//
// One item is a KV head of a request and up to 16 NQ of its (token, head of the
// group) rows.  The four waves of a workgroup take every fourth step of 32 keys
// with accumulators of their own and fold them at the end, so that every stored
// byte is loaded and converted once per item, whatever the number of rows.  Where
// there are more sequences than waves, and no long ones, a wave takes items of its
// own.
//
// Measured, 8 KV heads of 4 query heads, head dim 128: four requests' shares of 1M
// tokens, one row each and float32 O, 211 us for 1.14 GB, 5.4 TB/s, bound by HBM;
// 128 requests of 1 to 16K tokens 55 us for 0.23 GB, 4.2 TB/s, by the round trips
// at the ends of 1024 sequences; 2 x 1000 rows over 33K tokens 1016 us, 1.04
// PFLOP/s, by the instructions of a step of 64 rows and 32 keys: 64 matrix
// instructions of 16 cycles, 273 vector ones (32 exponentials, 64 conversions, 32
// permutes) of 4.5, or 9 while another wave's matrix instruction runs, 2400 cycles
// in all.  The same with float32 O, in tiles of 32 rows: 1892 us; 64 matrix and 282
// vector instructions a step, for half the rows.
//
// Under a score rule (mesh_attn_cache_score_fwd) a step's scores are capped, biased
// and put in log2 units between the products, rows see a range of keys, and a
// request's units begin at the first key that its rows see.  64 requests seen
// through windows of 4096 tokens, 8 KV heads of 4 query heads, head dim 128: 37 us,
// 3.1 TB/s, by the round trips of 512 sequences of 4 steps; 2 x 1000 rows over 16500
// keys with cap and bias 971 to 984 us, 0.53 PFLOP/s, by the vector unit (busy 0.73
// of the time, the matrix unit 0.22): tiles of 32 rows (a row's range, position and
// slope do not fit beside 64), twice the conversions, and a reciprocal and two
// exponentials per score.
//
// MFMA conventions (16x16x32): lane l holds, for A, row l % 16 and the k-values
// of quarter l / 16; for B, column l % 16 and the same quarter; accumulator
// register i holds row 4 (l / 16) + i of column l % 16.  The order of the
// k-values is free as long as A and B agree.  With r = l % 16, g = l / 16:
//  * K is A: row r of tile t (of two) is key 8 (r / 4) + 4 t + r % 4 of the
//    step, quarter g its dims g D/4 ..: one 16-byte load (8 at head dim 64).
//    The accumulators of the two tiles then hold the scores of keys 8 g .. 8 g
//    + 7, which is the k order that P as the second product's B operand needs:
//    no shuffle between the products.
//  * V^T is A: row r of MFMA m is dim r D/16 + m, quarter g the eight keys 8 g
//    ..: the cache keeps the D/16 dims of eight tokens together, 32 bytes (16)
//    per lane.  O's accumulators hold D/4 consecutive dims of a row per lane.
// The cache's conversion (two values an instruction, with the group's scale)
// gives pairs along the dims; a byte permute pairs keys for V.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_codes.h"
#include "tile_common.h"

namespace mesh_attn {
namespace {

using namespace dev;

constexpr int NT = 256;
constexpr int kWaves = NT / 64;
constexpr int kStep = 32;  // keys of a wave's step

__device__ __forceinline__ f32x4 mfma16(const bf16x8& a, const bf16x8& b,
                                        const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// x of the four lanes that share l % 16, joined by op.
template <typename Op>
__device__ __forceinline__ float across_quarters(float x, Op op) {
  x = op(x, __shfl_xor(x, 16));
  return op(x, __shfl_xor(x, 32));
}

// What a wave loads for a step: codes and scale codes of its lanes' keys.
template <int D>
struct StepData {
  uint32_t kc[2][D / 32];  // of a key's quarter
  uint32_t ks[2];
  uint32_t vc[D / 16];  // of a column's eight keys
  u32x2 vs;
};

// A request's keys of one KV head.  Everything but the lane's offsets is
// uniform over the wave.
struct Keys {
  const uint8_t* base;   // of the KV head in page 0
  const int32_t* table;  // the request's block table row
  int64_t page_bytes;    // from page to page
  int32_t lg, num_pages, last_page, local;
  // Offsets of the lane's operands in a step's first page (P16: in its page).
  uint32_t kc, ks, vc, vs;
};

// Pages of the two halves of the step at key kb (the same one unless a page is
// 16 tokens).  Scalar loads: the next step's numbers are there, without waiting
// for the vector loads in between, when its addresses are made.
struct StepPages {
  int32_t id[2];
};

template <bool P16>
__device__ __forceinline__ StepPages load_pages(const Keys& h, int kb) {
  StepPages s;
  const int at = kb >> h.lg;
  s.id[0] = load_const(h.table, min(at, h.last_page));
  s.id[1] = P16 ? load_const(h.table, min(at + 1, h.last_page)) : s.id[0];
  return s;
}

__device__ __forceinline__ bool valid_page(const Keys& h, int32_t id) {
  return id >= 0 && id < h.num_pages;
}

// The block of the page of half `second` of a step; page 0's for an invalid
// page, whose keys mask_step() hides.
template <bool P16>
__device__ __forceinline__ const uint8_t* page_block(const Keys& h,
                                                     const StepPages& pages,
                                                     bool second) {
  const int32_t i0 = valid_page(h, pages.id[0]) ? pages.id[0] : 0;
  const uint8_t* p0 = h.base + i0 * h.page_bytes;
  if (!P16) return p0;
  const int32_t i1 = valid_page(h, pages.id[1]) ? pages.id[1] : 0;
  const uint8_t* p1 = h.base + i1 * h.page_bytes;
  return second ? p1 : p0;
}

// Whether the page of the lane's keys 8 g .. 8 g + 7 of a step is valid.
template <bool P16>
__device__ __forceinline__ bool lane_ok(const Keys& h, const StepPages& pages,
                                        int g) {
  return valid_page(h, pages.id[P16 && g >= 2 ? 1 : 0]);
}

template <typename T>
__device__ __forceinline__ T load_at(const uint8_t* p) {
  return *reinterpret_cast<const T*>(p);
}

// Loads of K and of V of the step at key kb.  Keys past the end load bytes of
// the last page.
template <int D, bool P16>
__device__ __forceinline__ void load_k(const Keys& h, const StepPages& pages,
                                       int kb, int r, StepData<D>* s) {
  const uint8_t* kp = page_block<P16>(h, pages, r >= 8);
  // The step's first token in its page (0 with pages of 16).
  const uint32_t t0 = kb & ((1 << h.lg) - 1);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    // Offsets are summed in 32 bits: a scalar base and one register.
    const uint8_t* at = kp + (t0 * (D / 2) + h.kc + t * (4 * (D / 2)));
    if constexpr (D == 128) {
      const u32x4 w = load_at<u32x4>(at);
#pragma unroll
      for (int i = 0; i < 4; ++i) s->kc[t][i] = w[i];
    } else {
      const u32x2 w = load_at<u32x2>(at);
      s->kc[t][0] = w[0];
      s->kc[t][1] = w[1];
    }
    s->ks[t] = kp[t0 * (D / 32) + h.ks + t * (4 * (D / 32))];
  }
}

template <int D, bool P16>
__device__ __forceinline__ void load_v(const Keys& h, const StepPages& pages,
                                       int kb, int g, StepData<D>* s) {
  const uint8_t* vp = page_block<P16>(h, pages, g >= 2);
  const uint32_t t0 = kb & ((1 << h.lg) - 1);
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    const u32x4 w = load_at<u32x4>(vp + (t0 * (D / 2) + h.vc + 16 * j));
#pragma unroll
    for (int i = 0; i < 4; ++i) s->vc[4 * j + i] = w[i];
  }
  s->vs = load_at<u32x2>(vp + (t0 + h.vs));
}

// The lane's offsets for pages of 2^lg tokens.
template <int D>
__device__ __forceinline__ void lane_offsets(Keys* h, int r, int g) {
  using B = Block<D>;
  const int mask = (1 << h->lg) - 1;
  const int kt = (8 * (r >> 2) + (r & 3)) & mask, vt = (8 * g) & mask;
  h->kc = B::k_codes(h->lg, kt) + g * (D / 8);
  h->ks = B::k_scale(h->lg, kt, g * B::kGroups / 4);
  h->vc = B::v_codes(h->lg, vt, r);
  h->vs = B::v_scale(h->lg, vt, r * B::kGroups / 16);
}

// The item's rows and running state, 16 rows (columns of the MFMAs) per q.
//
// Up to 32 rows keep Q in registers; 64 rows would not fit beside O, and read it
// from LDS, in the order of the operand's lanes.
template <int NQ>
constexpr bool kQInLds = NQ > 2;

template <int D, int NQ>
struct State {
  bf16x8 q[kQInLds<NQ> ? 1 : NQ][D / 32];
  f32x4 o[NQ][D / 16];  // O^T, MFMA m of the lane's D/4 dims
  // Probabilities are 2^(score * scale - ref), with the reference at most kLag
  // below the row's running maximum; a score above `limit` moves it.  A row
  // without a finite score so far: limit -inf, neg_ref 0.
  float limit[NQ], neg_ref[NQ];
  float l[NQ];          // this lane's share of the sum
  int vis[NQ];          // stored keys that the column's row sees
};

// Under a score rule: keys [lo, vis) are seen, and the distance bias is taken
// relative to the nearest of them, `off` positions away, so that those of far keys
// keep their digits.
template <int NQ>
struct RuleState {
  int lo[NQ], qpos[NQ], off[NQ];
  float slope[NQ];  // log2 units
  // This lane's share of the sum of what the probabilities are rounded to (bf16
  // O): O is divided by it, so that the rounding of a row's largest ones falls out.
  float rounded[NQ];
  int before;       // stored keys that lie before all rows of the wave
};

// A row under the rule; of its request, the stored keys are [from, local).
struct RuleRow {
  int lo, vis, qpos, off, nearest;  // the key that `off` is the distance to
};

__device__ __forceinline__ int64_t key_position(const CacheFwdParams& p,
                                                int64_t key) {
  return p.c.share.striped ? key * p.c.share.n + p.c.share.p
                           : p.c.share.first + key;
}

__device__ __forceinline__ RuleRow rule_row(const CacheFwdParams& p,
                                            int64_t row, int from, int local) {
  RuleRow r;
  r.qpos = p.positions[row];
  const int64_t begin = p.key_begin ? max(p.key_begin[row], 0) : 0;
  const int64_t end =
      p.key_end ? max(p.key_end[row], 0) : int64_t{max(r.qpos, -1)} + 1;
  r.vis = min(p.c.share.below(end), local);
  r.lo = min(max(p.c.share.below(begin), from), r.vis);
  r.off = r.nearest = 0;
  if (p.slopes && r.lo < r.vis) {
    const int at = p.c.share.below(max(r.qpos, 0));  // first not before it
    const int64_t a = key_position(p, min(max(at, r.lo), r.vis - 1));
    const int64_t b = key_position(p, min(max(at - 1, r.lo), r.vis - 1));
    const int64_t da = a > r.qpos ? a - r.qpos : r.qpos - a;
    const int64_t db = b > r.qpos ? b - r.qpos : r.qpos - b;
    r.off = static_cast<int>(da < db ? da : db);
    r.nearest = min(max(da < db ? at : at - 1, r.lo), r.vis - 1);
  }
  return r;
}

// Products of a step -> scores in log2 units: capped (tanh(u) = 1 - 2 / (1 +
// e^(2u)); FINE: small arguments by its series) and biased.
template <bool FINE>
__device__ __forceinline__ float capped(const CacheFwdParams& p, float v,
                                        float add) {
  const float r =
      __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * p.cap_in));
  const float y = fmaf(-p.cap_two, r, fmaf(0.5f, p.cap_two, add));
  if (!FINE) return y;
  // Taylor; the first term left out is below 2^-23.9 of the sum.
  const float u = v * p.cap_u, z = u * u;
  float t = fmaf(z, -1382.f / 155925, 62.f / 2835);
  t = fmaf(t, z, -17.f / 315);
  t = fmaf(t, z, 2.f / 15);
  t = fmaf(t, z, -1.f / 3);
  t = fmaf(t * z, u, u);
  return fabsf(u) < 0.4f ? fmaf(t, 0.5f * p.cap_two, add) : y;
}

// Most positions from one stored key to the next for which the bias of a step is
// taken term by term: 2^-24 of 7 of them is below 2^-14, for slopes up to one.
constexpr int kNearSteps = 128;

template <int NQ, bool FINE>
__device__ __forceinline__ void rule_step(const CacheFwdParams& p,
                                          const RuleState<NQ>& rs,
                                          f32x4 (&x)[NQ][2], int kb, int g) {
  const int step = p.c.share.striped ? p.c.share.n : 1;
  const int k0 =
      p.slopes ? static_cast<int>(key_position(p, kb + 8 * g)) : 0;
  // In 32 bits: what wraps is not seen.
  const auto behind = [&](int q) {
    return static_cast<int>(static_cast<uint32_t>(rs.qpos[q]) -
                            static_cast<uint32_t>(k0));
  };
  // All keys before all rows: one more term per score.  (What the terms of eight
  // keys cancel is 2^-24 of 7 steps' bias: too much where keys lie far apart.)
  const bool before =
      p.slopes && kb + kStep <= rs.before && step <= kNearSteps;
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const float add =
        before ? -rs.slope[q] * static_cast<float>(behind(q) - rs.off[q]) : 0.f;
    if (p.cap_two > 0.f) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        x[q][i >> 2][i & 3] = capped<FINE>(p, x[q][i >> 2][i & 3], add);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        x[q][i >> 2][i & 3] = fmaf(x[q][i >> 2][i & 3], p.scale_log2, add);
    }
  }
  if (before) {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const float each = rs.slope[q] * static_cast<float>(step);
#pragma unroll
      for (int i = 1; i < 8; ++i)
        x[q][i >> 2][i & 3] =
            fmaf(each, static_cast<float>(i), x[q][i >> 2][i & 3]);
    }
  } else if (p.slopes) {
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int d = behind(q) - i * step;
        x[q][i >> 2][i & 3] =
            fmaf(-rs.slope[q],
                 static_cast<float>((d < 0 ? -d : d) - rs.off[q]),
                 x[q][i >> 2][i & 3]);
      }
  }
}

// The reference may lag behind the maximum by this much (log2 units):
// probabilities stay below 2^kLag, as exact relative to each other as below 1,
// and the accumulators are rescaled a few times per item instead of whenever a
// row's maximum grows.
constexpr float kLag = 8.f;

// Probabilities as the second product's operand.  For a bf16 O: rounded to
// bf16, 2^-8 of each, as O itself is.  For a float32 O: as the sum of three bf16
// that hold all 24 bits, cut off one after the other.
template <bool EXACT>
struct Probs {
  bf16x8 part[EXACT ? 3 : 1];
};

template <bool EXACT>
__device__ __forceinline__ void split_probs(const float (&p)[8],
                                            Probs<EXACT>* out) {
  if constexpr (EXACT) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p[i];
#pragma unroll
    for (int n = 0; n < 3; ++n) {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t lo = __float_as_uint(x[2 * i]);
        const uint32_t hi = __float_as_uint(x[2 * i + 1]);
        w[i] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
        x[2 * i] -= __uint_as_float(lo & 0xffff0000u);
        x[2 * i + 1] -= __uint_as_float(hi & 0xffff0000u);
      }
      out->part[n] = __builtin_bit_cast(bf16x8, w);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) out->part[0][i] = static_cast<__bf16>(p[i]);
  }
}

// The rest of a step once its scores x are there: keys 8 g + 4 t + i of column
// r.
template <int D, int NQ, bool EXACT, bool RULE>
__device__ __forceinline__ void finish_step(State<D, NQ>& st,
                                            RuleState<NQ>& rs,
                                            f32x4 (&x)[NQ][2],
                                            const StepData<D>& s,
                                            float scale_log2,
                                            float inv_scale_log2, u32x2 vs) {
  Probs<EXACT> ph[NQ];
  // One branch for all rows: it is rarely taken.
  float top[NQ];
  bool above = false;
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    top[q] = x[q][0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top[q] = fmaxf(top[q], x[q][i >> 2][i & 3]);
    above |= top[q] > st.limit[q];
  }
  if (__any(above)) {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const float t =
          across_quarters(top[q], [](float a, float b) { return fmaxf(a, b); }) *
          scale_log2;
      const bool none = st.limit[q] == -INFINITY;
      const float m = none ? t : fmaxf(-st.neg_ref[q], t);
      const bool still = !(m > -INFINITY);  // also for a NaN
      // Sums without a finite score so far are 0, or NaN.
      const float f =
          still || none ? 1.f : __builtin_amdgcn_exp2f(-st.neg_ref[q] - m);
      st.limit[q] = still ? -INFINITY
                          : fmaxf((m + kLag) * inv_scale_log2, -3e38f);
      st.neg_ref[q] = still ? 0.f : -m;
      st.l[q] *= f;
      if constexpr (RULE && !EXACT) rs.rounded[q] *= f;
#pragma unroll
      for (int m16 = 0; m16 < D / 16; ++m16) st.o[q][m16] *= f;
    }
  }
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      p[i] = __builtin_amdgcn_exp2f(
          fmaf(x[q][i >> 2][i & 3], scale_log2, st.neg_ref[q]));
    st.l[q] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    split_probs<EXACT>(p, &ph[q]);
    if constexpr (RULE && !EXACT)
      rs.rounded[q] = add_eight(ph[q].part[0], rs.rounded[q]);
  }
  float scale[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    scale[i] = scale_of((vs[i >> 2] >> (8 * (i & 3))) & 255u);
#pragma unroll
  for (int mp = 0; mp < D / 32; ++mp) {  // dims m = 2 mp and 2 mp + 1
    uint32_t pair[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // Key i's bytes: a word at head dim 128, half a word at 64.
      const uint32_t w = D == 128 ? s.vc[i] : s.vc[i >> 1];
      const int byte = D == 128 ? mp : 2 * (i & 1) + mp;
      bf16x2 v;
      switch (byte) {
        case 0: v = dequant2<0>(w, scale[i]); break;
        case 1: v = dequant2<1>(w, scale[i]); break;
        case 2: v = dequant2<2>(w, scale[i]); break;
        default: v = dequant2<3>(w, scale[i]); break;
      }
      pair[i] = __builtin_bit_cast(uint32_t, v);
    }
    u32x4 even, odd;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      even[i] = __builtin_amdgcn_perm(pair[2 * i + 1], pair[2 * i], 0x05040100u);
      odd[i] = __builtin_amdgcn_perm(pair[2 * i + 1], pair[2 * i], 0x07060302u);
    }
    const bf16x8 a0 = __builtin_bit_cast(bf16x8, even);
    const bf16x8 a1 = __builtin_bit_cast(bf16x8, odd);
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int n = 0; n < (EXACT ? 3 : 1); ++n) {
        st.o[q][2 * mp] = mfma16(a0, ph[q].part[n], st.o[q][2 * mp]);
        st.o[q][2 * mp + 1] = mfma16(a1, ph[q].part[n], st.o[q][2 * mp + 1]);
      }
  }
}

// A step in which some row of the item does not see some key, or a page is
// invalid: hidden scores are -inf, and V of keys that no column may use counts
// as 0.  A NaN group of V of a key that some rows see and others do not is taken
// out of the product (0 * NaN is NaN) and given to those that see it.
template <int D, int NQ, bool RULE>
__device__ __forceinline__ u32x2 mask_step(State<D, NQ>& st,
                                           const RuleState<NQ>& rs,
                                           f32x4 (&x)[NQ][2],
                                           const StepData<D>& s, bool ok,
                                           int kb, int local, int g) {
  u32x2 vs = s.vs;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (!ok || kb + 8 * g + i >= local) vs[i >> 2] &= ~(255u << (8 * (i & 3)));
#pragma unroll
  for (int q = 0; q < NQ; ++q)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!ok || kb + 8 * g + i >= st.vis[q] ||
          (RULE && kb + 8 * g + i < rs.lo[q]))
        x[q][i >> 2][i & 3] = -INFINITY;
  // Bit i: key 8 g + i of the lane's group of dims is NaN.
  uint32_t nan = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (((vs[i >> 2] >> (8 * (i & 3))) & 255u) == kScaleNaN) {
      nan |= 1u << i;
      vs[i >> 2] &= ~(255u << (8 * (i & 3)));
    }
  if (__any(nan != 0)) {
    // The lane's accumulators hold dims g D/4 ..: column n = 4 g is of their
    // group.
    bool hit[NQ] = {};
    for (int o = 0; o < 4; ++o) {  // keys 8 o ..
      const uint32_t bits = __shfl(nan, 16 * o + 4 * g);
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const int seen = min(max(st.vis[q] - (kb + 8 * o), 0), 8);
        uint32_t those = (1u << seen) - 1;
        if (RULE)
          those &= ~((1u << min(max(rs.lo[q] - (kb + 8 * o), 0), 8)) - 1);
        hit[q] |= (bits & those) != 0;
      }
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const float add = hit[q] ? NAN : 0.f;
#pragma unroll
      for (int m = 0; m < D / 16; ++m) st.o[q][m] += add;
    }
  }
  return vs;
}

// x = K Q^T of a step.  q_lds: Q in LDS, [q][c][lane].
template <int D, int NQ>
__device__ __forceinline__ void score_step(const State<D, NQ>& st,
                                           const bf16x8* q_lds,
                                           const StepData<D>& s, int lane,
                                           f32x4 (&x)[NQ][2]) {
  float sc[2];
#pragma unroll
  for (int t = 0; t < 2; ++t)
    sc[t] = s.ks[t] == kScaleNaN ? NAN : scale_of(s.ks[t]);
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    const bf16x8 a0 = dequant8(s.kc[0][c], sc[0]);
    const bf16x8 a1 = dequant8(s.kc[1][c], sc[1]);
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      if (c == 0) x[q][0] = x[q][1] = f32x4{0.f, 0.f, 0.f, 0.f};
      bf16x8 b;
      if constexpr (kQInLds<NQ>)
        b = q_lds[(q * (D / 32) + c) * 64 + lane];
      else
        b = st.q[q][c];
      x[q][0] = mfma16(a0, b, x[q][0]);
      x[q][1] = mfma16(a1, b, x[q][1]);
    }
  }
}

// One row's final results from its sums at reference m.
template <int D, bool OUT_F32, bool RULE>
__device__ __forceinline__ void store_row(const CacheFwdParams& p, int64_t row,
                                          int head, int from, int local,
                                          int dim0,
                                          const float (&acc)[8], float m,
                                          float l) {
  if (dim0 == 0) {
    if (RULE && p.slopes)  // the part of the bias that all keys share
      m -= p.slopes[head] * 1.4426950408889634f *
           static_cast<float>(rule_row(p, row, from, local).off);
    p.lse[int64_t{head} * p.rows + row] =
        l == 0.f ? -INFINITY
                 : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
  }
  const float inv = l > 0.f ? 1.f / l : l;  // 0 for no key; NaN stays
  const int64_t at = (row * p.hq + head) * D + dim0;
  if (OUT_F32) {
    f32x4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = acc[i] * inv;
      b[i] = acc[4 + i] * inv;
    }
    f32x4* dst = reinterpret_cast<f32x4*>(static_cast<float*>(p.o) + at);
    dst[0] = a;
    dst[1] = b;
  } else {
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = static_cast<__bf16>(acc[i] * inv);
    *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(p.o) + at) = v;
  }
}

// The token and the head (of all query heads) of row rr of a KV head's rows;
// group_mul / 2^group_shift is 1 / group, exact enough for rr < 2^30.
struct TokenHead {
  int tok, head;
};
__device__ __forceinline__ TokenHead token_head(const CacheFwdParams& p,
                                                uint32_t rr, int kvh) {
  const uint32_t tok = static_cast<uint32_t>(
      (uint64_t{rr} * p.group_mul) >> p.group_shift);
  return {int(tok), kvh * p.group + int(rr - tok * p.group)};
}

__device__ __forceinline__ int32_t stored_keys(const CacheFwdParams& p,
                                               int32_t len) {
  const int64_t most = int64_t{p.c.max_pages} << p.c.page_log2;
  const int64_t n = p.c.share.below(len < 0 ? 0 : len);
  return static_cast<int32_t>(n < most ? n : most);
}

// Work of a launch.  A sequence is a tile of a request's rows and a KV head; it
// is cut into units of 2^unit_log2 keys, a step of each wave or more (at least
// one unit, which writes the results of rows without keys).  All sequences'
// units in a row are dealt to the workgroups in equal runs of `per`, so every
// workgroup has the same work whatever the lengths, which only the device
// knows.  What a sequence costs beside its keys (finding it, the first loads, the
// fold) counts as seq_units units in front of them.  A sequence that lies in
// several runs leaves partial results, two slots a workgroup at most: slot 2 w
// for the piece that goes on from an earlier run, slot 2 w + 1 for the one that
// starts in run w and goes on after it; cache_fold_kernel joins them.  Not split:
// every sequence is one unit, and no piece is split.
constexpr int kWaveKeys = kWaves * kStep;  // keys of a step of each wave

// The factor that makes O's sums those of the unrounded probabilities' sum l.
template <int NQ, bool EXACT, bool RULE>
__device__ __forceinline__ float unrounded(const RuleState<NQ>& rs, int q,
                                           float l) {
  if constexpr (RULE && !EXACT) {
    const float r = across_quarters(
        rs.rounded[q], [](float a, float b) { return a + b; });
    return r > 0.f ? l / r : 1.f;
  }
  return 1.f;
}

// What the prefix sums leave in LDS per request: its first unit, and, for up to
// kKeptRequests requests, what an item needs (another round trip to memory
// otherwise).
constexpr int kKeptRequests = 256;

struct RequestRows {
  int first, end, local;
};
// Under a score rule no row sees the keys before `from`; the units of the
// request's sequences begin at the step that holds it.
struct RequestRule : RequestRows {
  int from;
};
template <bool RULE>
struct RequestOf {
  typedef RequestRows type;
};
template <>
struct RequestOf<true> {
  typedef RequestRule type;
};
template <bool RULE>
using Request = typename RequestOf<RULE>::type;

__device__ __forceinline__ int unit_keys(const RequestRows& r) {
  return r.local;
}
__device__ __forceinline__ int unit_keys(const RequestRule& r) {
  return r.local - (r.from & ~(kStep - 1));
}
__device__ __forceinline__ int first_key(const RequestRows&) { return 0; }
__device__ __forceinline__ int first_key(const RequestRule& r) {
  return r.from;
}

template <bool RULE>
__device__ __forceinline__ Request<RULE> load_request(const CacheFwdParams& p,
                                                      int b) {
  const int rows = static_cast<int>(p.rows);
  Request<RULE> r;
  const int a = p.cu[b], e = p.cu[b + 1];
  r.local = stored_keys(p, p.lens[b]);
  r.first = min(max(a, 0), rows);
  r.end = min(max(e, r.first), rows);
  if constexpr (RULE) {
    r.from = 0;
    if (p.key_begin && r.first < r.end)
      r.from = min(p.c.share.below(max(p.key_begin[r.first], 0)), r.local);
  }
  return r;
}

// A request's sequences: tiles of each KV head (none of a request that is another
// launch's), and units of each.
struct Sequences {
  int tiles, units;
};

template <int kRows, typename R>
__device__ __forceinline__ Sequences sequences_of(const CacheFwdParams& p,
                                                  const R& r, bool split) {
  const uint32_t rr = uint32_t(r.end - r.first) * p.group;  // below 2^30
  const bool mine = r.local >= p.least_keys && r.local <= p.most_keys;
  return {mine ? int((rr + kRows - 1) / kRows) : 0,
          split ? max((unit_keys(r) + (1 << p.unit_log2) - 1) >> p.unit_log2,
                      1)
                : 1};
}

// Whether the sequences of a launch that may cut them are better left whole,
// dealt out in turns: the cut gives every workgroup the same number of units, of
// which those that come after a tile's last row are none, and costs kCutUnits
// for the pieces of cut sequences and their fold; whole, the longest one and
// `turns` mean ones bound it, a mean one without half of the new keys.  An
// estimate: rows may see less or more than this.  Microseconds cut / whole, 8 KV
// heads of 4:
//   1 x 4000 of 4000 keys  244/157    2 x 1000 of 33000  1018/968
//   1 x  900 of 2000        57/38     1 x 1100 of 20000   352/484
//   1 x  130 of 2000        28/33     1 x  900 of 20000   294/300
constexpr int kCutUnits = 10;

struct Totals {
  unsigned long long seqs, units, mean;
  int longest;
};

template <int kRows, bool RULE>
__device__ __forceinline__ bool whole_is_better(const CacheFwdParams& p,
                                                Totals* s_totals) {
  if (threadIdx.x == 0) *s_totals = Totals{0, 0, 0, 0};
  __syncthreads();
  for (int b = threadIdx.x; b < p.num_requests; b += NT) {
    const Request<RULE> r = load_request<RULE>(p, b);
    const Sequences q = sequences_of<kRows>(p, r, true);
    if (q.tiles == 0) continue;
    const int64_t n = int64_t{q.tiles} * p.c.hkv;
    const int all = q.units + p.seq_units;
    // The keys of the new rows, if they are the request's last positions.
    const int fresh =
        r.local - stored_keys(p, max(p.lens[b], 0) - (r.end - r.first));
    const int mean = all - min(fresh >> (p.unit_log2 + 1), all - 1);
    atomicAdd(&s_totals->seqs, static_cast<unsigned long long>(n));
    atomicAdd(&s_totals->units, static_cast<unsigned long long>(n * all));
    atomicAdd(&s_totals->mean, static_cast<unsigned long long>(n * mean));
    atomicMax(&s_totals->longest, all);
  }
  __syncthreads();
  const uint64_t n = s_totals->seqs, grid = gridDim.x;
  const uint64_t cut = s_totals->units / grid + kCutUnits;
  const uint64_t turns = (n + grid - 1) / grid;
  return uint64_t(s_totals->longest) <= cut &&
         turns * s_totals->mean <= cut * n;
}

// First units of the requests in LDS, by prefix sums over the workgroup; the
// sums are capped at max_units, which rows that do not overlap cannot pass.
// Returns the number of units; *longest is the longest sequence of a request
// with several tiles (0: there is none).
template <int kRows, bool RULE>
__device__ __forceinline__ int plan_units(const CacheFwdParams& p, bool split,
                                          int* s_units, Request<RULE>* s_kept,
                                          int* s_wave, int* s_longest,
                                          int* longest) {
  const int B = p.num_requests, tid = threadIdx.x, lane = tid & 63;
  const int cost = split ? p.seq_units : 0;
  int base = 0;
  if (tid == 0) *s_longest = 0;
  __syncthreads();
  for (int b0 = 0; b0 < B; b0 += NT) {
    const int b = b0 + tid;
    int mine = 0;
    if (b < B) {
      const Request<RULE> r = load_request<RULE>(p, b);
      if (B <= kKeptRequests) s_kept[b] = r;
      const Sequences q = sequences_of<kRows>(p, r, split);
      const int64_t n = int64_t{q.tiles} * (q.units + cost) * p.c.hkv;
      mine = static_cast<int>(n < p.max_units ? n : p.max_units);
      if (kRows > 16 && q.tiles > 1) atomicMax(s_longest, q.units + cost);
    }
    int y = mine;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int z = __shfl_up(y, o);
      if (lane >= o) y = min(y + z, p.max_units);
    }
    int before = __shfl_up(y, 1);  // every lane takes part
    if (lane == 0) before = 0;
    if (lane == 63) s_wave[tid >> 6] = y;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < (tid >> 6)) before = min(before + s_wave[w], p.max_units);
    }
    if (b < B) s_units[b] = min(base + before, p.max_units);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) base = min(base + s_wave[w], p.max_units);
    __syncthreads();
  }
  if (tid == 0) s_units[B] = base;
  __syncthreads();
  *longest = *s_longest;
  return base;
}

// The thread's index, not known to be the same from call to call: what is
// derived from it is computed where it is used instead of being held in
// registers through the loop over the keys.
__device__ __forceinline__ int fresh_tid() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// Waves per SIMD: as many as the registers allow with few spills.  Head dim 128,
// 16 rows: 3 (768 workgroups) read 1.1 GB in 209 us, 4 with spills 239; 32 rows:
// 2 took 80 us for 16 requests of 8 tokens of 4 heads over 16K tokens (68 now, where
// the bytes take 53), 3 with spills 127.  64 rows at head dim 128 spill with 2: where
// sequences are cut 6 registers, around the loop over the keys, or with pages of 16
// 20, of which a step reads 5; where waves own theirs 2 and 3.
template <int D, int NQ>
constexpr int kWavesPerSimd = D == 64 ? (NQ == 1 ? 4 : NQ == 2 ? 3 : 2)
                                      : (NQ == 1 ? 3 : 2);

// An item of a workgroup: units [u0, u1) of the nu of a sequence (none if the
// run ends before the keys), the last of them before `end` in all units.
struct Item {
  int b, first, rr0, rr_end, kvh, u0, u1, nu, local, end;
  int from, skip;  // first key; keys before the first unit
};

// The item at unit `at` of a run that ends at `stop`.
template <int kRows, bool OWN, bool RULE>
__device__ __forceinline__ Item locate(const CacheFwdParams& p, bool split,
                                       const int* s_units,
                                       const Request<RULE>* s_kept, int at,
                                       int stop) {
  const int B = p.num_requests, hkv = p.c.hkv;
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (s_units[mid] <= at)
      lo = mid;
    else
      hi = mid;
  }
  Item it;
  it.b = __builtin_amdgcn_readfirstlane(lo);
  const Request<RULE> req =
      B <= kKeptRequests ? s_kept[it.b] : load_request<RULE>(p, it.b);
  it.first = __builtin_amdgcn_readfirstlane(req.first);
  it.rr_end = __builtin_amdgcn_readfirstlane(req.end - req.first) * p.group;
  it.local = __builtin_amdgcn_readfirstlane(req.local);
  it.from = RULE ? __builtin_amdgcn_readfirstlane(first_key(req)) : 0;
  it.skip = it.from & ~(kStep - 1);
  it.nu = split ? max((it.local - it.skip + (1 << p.unit_log2) - 1) >>
                          p.unit_log2,
                      1)
                : 1;
  const int off = at - __builtin_amdgcn_readfirstlane(s_units[it.b]);
  const int len = split ? it.nu + p.seq_units : 1, seq = off / len;
  const int v0 = off - seq * len;  // of the sequence's units with its cost
  it.u0 = split ? max(v0 - p.seq_units, 0) : 0;
  it.u1 = split ? min(v0 + (stop - at) - p.seq_units, it.nu) : 1;
  it.end = min(at - v0 + len, stop);
  const int tiles = (it.rr_end + kRows - 1) / kRows;
  int tile;
  if (OWN) {
    // The waves of a workgroup take neighbouring tiles of a head, and the next
    // workgroups, which run on other XCDs, the same tiles of the next heads.
    // Causal rows: the last tiles, which see the most keys, come first.
    const int quad = seq / (kWaves * hkv), rest = seq - quad * (kWaves * hkv);
    const int n = min(kWaves, tiles - quad * kWaves);
    it.kvh = rest / n;
    tile = tiles - 1 - (quad * kWaves + rest - it.kvh * n);
  } else if (split) {
    // Runs of neighbouring tiles of a head read the same keys.
    it.kvh = seq / tiles;
    tile = seq - it.kvh * tiles;
  } else {
    // Workgroup i runs on XCD i % 8: with a multiple of 8 heads, a head's keys
    // are read through one L2.
    const int from_last = seq / hkv;
    it.kvh = seq - from_last * hkv;
    tile = tiles - 1 - from_last;
  }
  it.rr0 = tile * kRows;
  return it;
}

// OWN: every wave has items of its own, whole sequences, and nothing to fold.
// RULE: scores under a rule (mesh_attn_cache_score_fwd).  FINE: the tanh of small
// arguments by its series (a float32 O, and wide caps: as a branch of the step it
// took 2 % of a chunk under a usual cap at head dim 128, 6 % at 64).
template <int D, int NQ, bool OUT_F32, bool P16, bool OWN, bool RULE, bool FINE>
__global__ __launch_bounds__(NT, (kWavesPerSimd<D, NQ>))
void cache_fwd_kernel(CacheFwdParams p) {
  constexpr int kRows = 16 * NQ;
  constexpr int kPad = D + 4;  // row stride of the fold, in floats
  constexpr int kFolded = OWN ? 1 : kWaves;
  constexpr int kQ = NQ * (D / 32) * 64;
  __shared__ float s_o[kFolded][16][kPad];
  __shared__ float s_m[kFolded][16], s_l[kFolded][16];
  __shared__ bf16x8 s_q_all[kQInLds<NQ> ? (OWN ? kWaves : 1) * kQ : 1];
  __shared__ int s_wave[kWaves], s_longest;
  extern __shared__ int s_units[];  // [B + 1], then the kept requests
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, g = lane >> 4;
  Request<RULE>* s_kept =
      reinterpret_cast<Request<RULE>*>(s_units + p.num_requests + 1);
  bf16x8* s_q = s_q_all + (OWN && kQInLds<NQ> ? wave * kQ : 0);
  bool split = !OWN && p.split;
  if constexpr (kRows > 16 && !OWN) {
    __shared__ Totals s_totals;
    if (split && p.may_stay_whole)
      split = !__builtin_amdgcn_readfirstlane(
          whole_is_better<kRows, RULE>(p, &s_totals));
  }

  int longest;
  const int total = __builtin_amdgcn_readfirstlane(
      plan_units<kRows, RULE>(p, split, s_units, s_kept, s_wave, &s_longest,
                              &longest));
  // Split: this workgroup's run.  Workgroup i runs on XCD i % 8; neighbouring
  // runs go to one XCD (the grid is a multiple of 8), whose L2 then serves the
  // tiles of a head, and the runs with work spread over all of them.
  int run = blockIdx.x, per = 1, stop = total;
  int at = OWN ? run * kWaves + wave : run;
  // Whole sequences: to the workgroup's next one; where tiles differ, there and
  // back again, so that those with the longer ones of one turn have the shorter
  // ones of the next.
  constexpr bool kBack = kRows > 16 && !OWN;
  int hop = kBack ? 2 * int(gridDim.x - 1 - run) + 1
                  : int(gridDim.x) * (OWN ? kWaves : 1);
  if (split) {
    per = max((total + int(gridDim.x) - 1) / int(gridDim.x), 1);
    if (kRows > 16 && longest > 0) {
      // Whole sequences per run, where that costs at most a twentieth: the tiles
      // of a head then walk over the keys side by side, and find them in their
      // L2.  1000 rows of 4 heads a request over 33K tokens, when cut: 30 million
      // misses and 1103 us without, 2 million and 1037 us with.
      longest = __builtin_amdgcn_readfirstlane(longest);
      const int whole = (per + longest - 1) / longest * longest;
      if (whole - per <= per / 20) per = whole;
    }
    const int active = (total + per - 1) / per;
    const int each = (active + 7) / 8;  // of an XCD
    const int x = blockIdx.x % 8, y = blockIdx.x / 8;
    // The others take the runs behind the active ones, without work.
    run = y < each ? x * each + y
                   : 8 * each + x * (int(gridDim.x / 8) - each) + y - each;
    // Below 2^31: total is below 2^30, and per * gridDim at most a twentieth
    // and two gridDim larger.
    at = per * run;
    stop = min(at + per, total);
  }
  if (!OWN && p.split && tid == 0)
    p.fold[2 * run].parts = p.fold[2 * run + 1].parts = 0;

  State<D, NQ> st;
  RuleState<NQ> rs;
  Item it, prev;
  bool have_prev = false;
  for (;;) {
    bool more = false;
    while (at < stop && !more) {
      it = locate<kRows, OWN, RULE>(p, split, s_units, s_kept, at, stop);
      if (split) {
        at = it.end;
      } else {
        at += hop;
        if (kBack) hop = 2 * int(gridDim.x) - hop;
      }
      more = it.u0 < it.u1;
    }
    Keys h;
    StepPages pg;
    StepData<D> s;
    int pos[NQ], kb = 0, piece_end = 0;
    if (more) {
      // The first step's loads go out with those of Q and the positions, and
      // all of them before the last item's fold.
      h.lg = p.c.page_log2;
      h.num_pages = p.c.num_pages;
      h.table = p.block_table + int64_t{it.b} * p.c.max_pages;
      h.local = it.local;
      h.last_page = max((it.local - 1) >> h.lg, 0);
      h.page_bytes = int64_t{p.c.hkv} * p.c.block_bytes();
      h.base = p.data + int64_t{it.kvh} * p.c.block_bytes();
      lane_offsets<D>(&h, r, g);
      kb = (split ? it.u0 << p.unit_log2 : 0) + (OWN ? 0 : wave * kStep);
      piece_end = split ? min(int64_t{it.u1} << p.unit_log2,
                              int64_t{it.local})
                        : it.local;
      if constexpr (RULE) {
        kb += it.skip;
        if (split)
          piece_end = min((int64_t{it.u1} << p.unit_log2) + it.skip,
                          int64_t{it.local});
      }
      pg = load_pages<P16>(h, kb);
      if (kQInLds<NQ> && !OWN) lds_barrier();  // the last item's Q has been read
      const int t = fresh_tid(), r = t & 15, g = (t & 63) >> 4, lane = t & 63;
      bf16x8 staged[kQInLds<NQ> && OWN ? NQ : 1][D / 32];  // to LDS later
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const int mine = it.rr0 + 16 * q + r;
        const uint32_t rr = mine < it.rr_end ? mine : it.rr0;
        const TokenHead th = token_head(p, rr, it.kvh);
        const int64_t row = int64_t{it.first} + th.tok;
        const uint16_t* src =
            p.q + row * p.q_stride + int64_t{th.head} * D + g * (D / 4);
        pos[q] = p.positions[row];
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          if constexpr (!kQInLds<NQ>)
            st.q[q][c] = *reinterpret_cast<const bf16x8*>(src + 8 * c);
          else if constexpr (OWN)
            staged[q][c] = *reinterpret_cast<const bf16x8*>(src + 8 * c);
          else if (q % kWaves == wave)
            s_q[(q * (D / 32) + c) * 64 + lane] =
                *reinterpret_cast<const bf16x8*>(src + 8 * c);
        }
      }
      if (kb < piece_end) {
        load_k<D, P16>(h, pg, kb, r, &s);
        load_v<D, P16>(h, pg, kb, g, &s);
      }
      if constexpr (kQInLds<NQ> && OWN) {
#pragma unroll
        for (int q = 0; q < NQ; ++q)
#pragma unroll
          for (int c = 0; c < D / 32; ++c)
            s_q[(q * (D / 32) + c) * 64 + lane] = staged[q][c];
      }
    }

    if constexpr (!OWN) if (have_prev) {
      // Fold the waves, 16 rows at a time.
      const bool whole = prev.u0 == 0 && prev.u1 == prev.nu;
      const int slot = 2 * run + (prev.u0 == 0 ? 1 : 0);
      const int tid = fresh_tid(), r = tid & 15, g = (tid & 63) >> 4;
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        if (prev.rr0 + 16 * q >= prev.rr_end) break;
        const float l = across_quarters(
            st.l[q], [](float a, float b) { return a + b; });
        const float factor = unrounded<NQ, OUT_F32, RULE>(rs, q, l);
        lds_barrier();
        if (g == 0) {
          s_m[wave][r] =
              st.limit[q] == -INFINITY ? -INFINITY : -st.neg_ref[q];
          s_l[wave][r] = l;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int m = 0; m < D / 16; ++m)
            s_o[wave][r][g * (D / 4) + i * (D / 16) + m] =
                RULE && !OUT_F32 ? st.o[q][m][i] * factor : st.o[q][m][i];
        lds_barrier();
        const int row16 = tid / (D / 8), dim0 = tid % (D / 8) * 8;
        const int rr = prev.rr0 + 16 * q + row16;
        if (row16 < 16 && rr < prev.rr_end) {
          float M = -INFINITY;
#pragma unroll
          for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_m[w][row16]);
          const float ref = M == -INFINITY ? 0.f : M;
          float L = 0.f, acc[8] = {};
#pragma unroll
          for (int w = 0; w < kWaves; ++w) {
            // A wave without a finite score has sums of 0, or of NaN.
            const float sm = s_m[w][row16] == -INFINITY
                                 ? 1.f
                                 : __builtin_amdgcn_exp2f(s_m[w][row16] - ref);
            L += s_l[w][row16] * sm;
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] += s_o[w][row16][dim0 + i] * sm;
          }
          if (whole) {
            const TokenHead th = token_head(p, rr, prev.kvh);
            store_row<D, OUT_F32, RULE>(p, prev.first + th.tok, th.head,
                                        prev.from, prev.local, dim0, acc, ref,
                                        L);
          } else {
            const int64_t pr = int64_t{slot} * kRows + 16 * q + row16;
            if (dim0 == 0) {
              p.part_ml[2 * pr] = M;
              p.part_ml[2 * pr + 1] = L;
            }
            f32x4* dst = reinterpret_cast<f32x4*>(p.part_o + pr * D + dim0);
            dst[0] = f32x4{acc[0], acc[1], acc[2], acc[3]};
            dst[1] = f32x4{acc[4], acc[5], acc[6], acc[7]};
          }
        }
      }
    }
    if (!more) break;

    int most_seen = 0, all_see = INT32_MAX, all_from = 0;
    if (RULE) rs.before = INT32_MAX;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int r = fresh_tid() & 15;
      const bool valid = it.rr0 + 16 * q + r < it.rr_end;
      bool sure = true;  // the nearest key is there
      if constexpr (RULE) {
        const uint32_t rr = valid ? it.rr0 + 16 * q + r : it.rr0;
        const TokenHead th = token_head(p, rr, it.kvh);
        const RuleRow row =
            rule_row(p, int64_t{it.first} + th.tok, it.from, it.local);
        st.vis[q] = valid ? row.vis : 0;
        rs.lo[q] = row.lo;
        rs.qpos[q] = row.qpos;
        rs.off[q] = row.off;
        rs.slope[q] =
            p.slopes ? p.slopes[th.head] * 1.4426950408889634f : 0.f;
        if (p.slopes && row.lo < row.vis)
          sure = valid_page(h, h.table[row.nearest >> h.lg]);
        if (valid) {
          all_from = max(all_from, row.lo);
          rs.before =
              min(rs.before, p.c.share.below(int64_t{max(row.qpos, -1)} + 1));
        }
      } else {
        st.vis[q] = valid ? min(p.c.share.below(int64_t{max(pos[q], -1)} + 1),
                                it.local)
                          : 0;
      }
      most_seen = max(most_seen, st.vis[q]);
      if (valid) all_see = min(all_see, st.vis[q]);
      st.limit[q] = -INFINITY;
      st.neg_ref[q] = st.l[q] = 0.f;
      if (RULE) rs.rounded[q] = 0.f;
      // Under a moderate cap, with a bias that falls, the largest probability
      // lies between 2^-kLow and 2^40 around a fixed reference (1, where twice the
      // cap fits in kLow), and what a bias leaves of others is a normal number down
      // to 2^-21 of it.  (A float32 O's third parts are 2^16 smaller.)
      constexpr float kLow = OUT_F32 ? 100.f : 105.f;
      if (RULE && p.cap_two > 0.f && p.cap_two <= kLow + 40.f &&
          !(rs.slope[q] < 0.f) && sure) {
        st.limit[q] = INFINITY;
        st.neg_ref[q] = -fminf(0.5f * p.cap_two, kLow - 0.5f * p.cap_two);
      }
#pragma unroll
      for (int m = 0; m < D / 16; ++m) st.o[q][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int o = 1; o < 16; o *= 2) {
      most_seen = max(most_seen, __shfl_xor(most_seen, o));
      all_see = min(all_see, __shfl_xor(all_see, o));
      if (RULE) {
        all_from = max(all_from, __shfl_xor(all_from, o));
        rs.before = min(rs.before, __shfl_xor(rs.before, o));
      }
    }
    most_seen = __builtin_amdgcn_readfirstlane(most_seen);
    all_see = __builtin_amdgcn_readfirstlane(all_see);
    if (RULE) {
      all_from = __builtin_amdgcn_readfirstlane(all_from);
      rs.before = __builtin_amdgcn_readfirstlane(rs.before);
    }
    if (kQInLds<NQ> && !OWN) lds_barrier();

    // The next step's K is loaded into the registers of this one's as soon as
    // the first product has read them, its V after the second: each is in
    // flight for about half a step, without registers of its own.
    const int kend = min(piece_end, most_seen);
    if (kb < kend) {
      for (;;) {
        const int next = kb + (OWN ? kStep : kWaveKeys);
        const bool more_keys = next < kend;
        const StepPages pn = load_pages<P16>(h, next);
        // Q's LDS reads stay in the loop (its registers are needed).
        if constexpr (kQInLds<NQ>) asm volatile("" ::: "memory");
        f32x4 x[NQ][2];
        // The wave with matrix instructions to issue goes first: the other
        // waves' vector work fits between them.
        __builtin_amdgcn_s_setprio(1);
        score_step<D, NQ>(st, s_q, s, lane, x);
        __builtin_amdgcn_s_setprio(0);
        if (more_keys) load_k<D, P16>(h, pn, next, r, &s);
        u32x2 vs = s.vs;
        const bool ok = lane_ok<P16>(h, pg, g);
        if constexpr (RULE) rule_step<NQ, FINE>(p, rs, x, kb, g);
        if (kb + kStep > all_see || (RULE && kb < all_from) || !__all(ok))
          vs = mask_step<D, NQ, RULE>(st, rs, x, s, ok, kb, h.local, g);
        finish_step<D, NQ, OUT_F32, RULE>(st, rs, x, s,
                                          RULE ? 1.f : p.scale_log2,
                                          RULE ? 1.f : p.inv_scale_log2, vs);
        if (!more_keys) break;
        load_v<D, P16>(h, pn, next, g, &s);
        pg = pn;
        kb = next;
      }
    }

    if constexpr (OWN) {
      // Stored before the next item's loads, which then have its registers.
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const int tid = fresh_tid(), r = tid & 15, g = (tid & 63) >> 4;
        if (it.rr0 + 16 * q >= it.rr_end) continue;
        const float l = across_quarters(
            st.l[q], [](float a, float b) { return a + b; });
        const float factor = unrounded<NQ, OUT_F32, RULE>(rs, q, l);
        const int rr = it.rr0 + 16 * q + r;
        const TokenHead th = token_head(p, rr, it.kvh);
        if (rr < it.rr_end) {
#pragma unroll
          for (int j = 0; j < D / 32; ++j) {
            float acc[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
              acc[i] = st.o[q][(8 * j + i) % (D / 16)][(8 * j + i) / (D / 16)] *
                       (RULE && !OUT_F32 ? factor : 1.f);
            store_row<D, OUT_F32, RULE>(
                p, it.first + th.tok, th.head, it.from, it.local,
                g * (D / 4) + 8 * j, acc,
                st.limit[q] == -INFINITY ? 0.f : -st.neg_ref[q], l);
          }
        }
      }
    }
    const bool goes_on = it.u0 > 0;  // then it is the run's first item
    if (split && (goes_on || it.u1 < it.nu) && tid == 0) {
      // The runs that the sequence's keys lie in; the rest of them fill runs
      // from this one's start or, if they start here, after its end.
      CacheFold f;
      f.first = it.first;
      f.rr0 = it.rr0;
      f.rr_end = it.rr_end;
      f.kvh = it.kvh;
      f.start = goes_on ? (per * run - it.u0) / per : run;
      const int more_runs = goes_on ? (it.nu - it.u0 - 1) / per
                                    : (it.nu - it.u1 + per - 1) / per;
      f.parts = min(run + more_runs, int(gridDim.x) - 1) - f.start + 1;
      p.fold[2 * run + (goes_on ? 0 : 1)] = f;
      if (RULE)
        p.fold_keys[2 * run + (goes_on ? 0 : 1)] = {it.from, it.local};
    }
    prev = it;
    have_prev = true;
  }
}

// Joins the partial results of the sequences that several runs hold: slots 2 w +
// 1, 2 (w + 1), 2 (w + 2), .. of the one that starts in run w, in an order of
// their own, whatever order they were made in.  The workgroups of its runs take
// a slice of its rows each, down to one row; eight dims per thread, and as many
// threads per row as there are take turns at the pieces and join through LDS.
// Both launches, so / with one workgroup per sequence: 34 requests of 1 to 56K
// tokens of one head 17/46 us, 2 of 51K 19/56 us.
constexpr int kFoldThreads = 512;

template <int D, int NQ, bool OUT_F32, bool RULE>
__global__ __launch_bounds__(kFoldThreads)
void cache_fold_kernel(CacheFwdParams p) {
  constexpr int kRows = 16 * NQ, kDimThreads = D / 8;
  __shared__ float s_acc[kFoldThreads][9];  // [9]: apart in the LDS banks
  __shared__ float s_m[kFoldThreads / kDimThreads];
  __shared__ float s_l[kFoldThreads / kDimThreads];
  const int run = blockIdx.x, tid = threadIdx.x;
#pragma unroll 1
  for (int which = 0; which < 2; ++which) {
    const CacheFold f = load_const(p.fold, 2 * run + which);
    CacheFoldKeys keys = {0, 0};  // (of no use without a sequence)
    if (RULE) keys = load_const(p.fold_keys, 2 * run + which);
    if (f.parts < 2) continue;
    // Rows of a slice; more than one run, so they are half of all at most.
    int n = kRows / 2;
    while (n > 1 && kRows / n * 2 <= f.parts) n /= 2;
    const int q0 = (run - f.start) * n;
    if (q0 >= kRows || f.rr0 + q0 >= f.rr_end) continue;
    const int dim0 = tid % kDimThreads * 8;
    const int at = tid / kDimThreads, my = at % n, pg = at / n;
    const int groups = kFoldThreads / (n * kDimThreads);  // a power of two
    const int row = q0 + my, rr = f.rr0 + row;
    const bool valid = rr < f.rr_end;
    float M = -INFINITY, L = 0.f, acc[8] = {};
    auto fold = [&](float m, float l, const float* x) {
      const float mn = fmaxf(M, m);
      const float ref = mn == -INFINITY ? 0.f : mn;
      const float a = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(M - ref);
      const float b = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - ref);
      L = L * a + l * b;
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] = acc[i] * a + x[i] * b;
      M = mn;
    };
    if (valid)
#pragma unroll 4
      for (int i = pg; i < f.parts; i += groups) {
        const int64_t w = f.start + i;
        const int64_t pr = (i == 0 ? 2 * w + 1 : 2 * w) * kRows + row;
        float x[8];
        const f32x4* src =
            reinterpret_cast<const f32x4*>(p.part_o + pr * D + dim0);
        const f32x4 lo = src[0], hi = src[1];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[j] = lo[j];
          x[4 + j] = hi[j];
        }
        fold(p.part_ml[2 * pr], p.part_ml[2 * pr + 1], x);
      }
    for (int half = groups / 2; half > 0; half /= 2) {
      if (half >= f.parts) continue;
      __syncthreads();
      if (pg >= half && pg < 2 * half) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s_acc[tid][i] = acc[i];
        s_m[at] = M;  // the same of all dims' threads
        s_l[at] = L;
      }
      __syncthreads();
      if (pg < half)
        fold(s_m[at + half * n], s_l[at + half * n],
             s_acc[tid + half * n * kDimThreads]);
    }
    if (pg == 0 && valid) {
      const TokenHead th = token_head(p, rr, f.kvh);
      store_row<D, OUT_F32, RULE>(p, f.first + th.tok, th.head, keys.from,
                                  keys.local, dim0, acc,
                                  M == -INFINITY ? 0.f : M, L);
    }
    __syncthreads();
  }
}

// Workgroups that fit the card at once: each has a wave on every SIMD of one of
// 256 compute units.
int resident_groups(int head_dim, int nq) {
  if (head_dim == 64)
    return 256 * (nq == 1   ? kWavesPerSimd<64, 1>
                  : nq == 2 ? kWavesPerSimd<64, 2>
                            : kWavesPerSimd<64, 4>);
  return 256 * (nq == 1   ? kWavesPerSimd<128, 1>
                : nq == 2 ? kWavesPerSimd<128, 2>
                          : kWavesPerSimd<128, 4>);
}

// How a call is launched, from its sizes alone: requests of up to own_keys stored
// keys with a wave for every sequence (-1: none), the others cut, or, without
// `cut`, with a workgroup for every sequence.
struct Shape {
  int nq;  // 16-row columns per tile
  bool cut, may_stay_whole;  // .. where the device finds it better
  int own_keys, own_grid, whole_grid, cut_grid;
  int unit_log2, max_units;
};

// Units that a sequence counts beside its keys.  128 requests of 1 to 16384
// tokens (half of them shorter than a unit), 8 KV heads, keys in the last-level
// cache / not: 82 us with 0, 50/58 with 2, 48/61 with 4, -/71 with 12; requests
// of one length take the same within 4 %.
constexpr int kSeqUnits = 2;

// Most stored keys of a request, and how many of them are always one launch's.
int64_t keys_of(const CacheDims& c) {
  return int64_t{c.max_pages} << c.page_log2;
}
constexpr int64_t kBriefKeys = 512;

// Workgroups of a launch of whole sequences per wave, of what fits at once: more
// are dealt out as others end, each makes the plan.  4 x 4000 rows of 4 heads and
// as many keys: 633 us with 2, 527 with 4 and with 8; 106 x 444 of 16: 1257, 1276
// and 1296.
constexpr int64_t kOwnGrid = 4;

Shape shape_of(const CacheDims& c, int32_t hq, int32_t num_requests,
               int64_t rows, bool out_f32, bool rule) {
  const int group = hq / c.hkv;
  Shape s;
  // Rows of a request, were they all alike: the host knows no more.  A batch of
  // decode tokens and a chunk has one height for both: 127 requests of a token and
  // one of 300 over 16K keys (16 rows) take 199 us, apart 47 and 107.
  const int64_t each = (rows + num_requests - 1) / num_requests * group;
  // Three bf16 parts of 64 rows' probabilities do not fit the registers: 1000
  // rows of 4 heads over 33K tokens take 1894 us in tiles of 32 rows, 2175 of 64.
  // Under a rule neither do a row's range, position and slope at head dim 128 (70
  // to 110 registers in memory: 2 x 1000 rows of 4 heads over 16500 keys with cap
  // and bias take 1610 us in tiles of 64 rows, 1180 of 32).
  s.nq = each <= 16                                         ? 1
         : each <= 32 || out_f32 || (rule && c.d == 128) ? 2
                                                            : 4;
  // Most sequences that rows which do not overlap make.
  const int64_t seqs = (rows * group / (16 * s.nq) + num_requests) * c.hkv;
  const int slots = resident_groups(c.d, s.nq);
  const int64_t keys = keys_of(c);
  // Short tables are not worth a second launch.  (The lengths may be shorter still,
  // which the host cannot know: wide tables of short requests are cut.)
  // Microseconds cut / whole, one row of 4 heads per KV head, 8 KV heads:
  //   1 request of 256 tokens  9.1/6.7   64 of  512   18.3/12.1
  //   1 of 1024               10.0/11.6  64 of 1024   22.0/17.3
  //   1 of 2048               10.4/16.4  32 of 1..1024 13.5/11.4
  const bool brief = keys <= kBriefKeys || (keys <= 1024 && seqs >= 256);
  const bool one_tile = each <= 16 * s.nq;
  // A wave each for whole sequences, where there are enough for all waves and
  // the last round of them is nearly full: nothing is folded, and a wave's own
  // overhead lies beside the others' work.  Microseconds so / a workgroup each,
  // 8 KV heads:
  //   106 x 444 rows of 16 heads    1276/3145   8 x 600 rows of 4 heads over 4096
  //   16 x 600 of 4, float32 O       135/237    (2464 for 2048 waves)  411/329
  //   1000 x 1 of 4, 1 to 500 keys    47/107    8 x 2000 of 2000       331/419
  // Requests with far more keys than rows are not among them (nor are those of one
  // tile): a few of them would be a few waves' work, long after the others.
  const int64_t waves = int64_t{kWaves} * slots;
  const int64_t rounds = (seqs + waves - 1) / waves;
  const bool own = (brief || !one_tile) && seqs >= waves &&
                   (rounds > 2 || rounds * waves - seqs <= seqs / 4);
  const int64_t tokens = (rows + num_requests - 1) / num_requests;
  const int64_t limit = tokens < 1024 ? 2048 : 2 * tokens;
  s.own_keys = !own ? -1
                    : static_cast<int>(brief || limit > keys ? keys : limit);
  // The others, unless tables are short, are cut, or left whole by workgroups
  // where the lengths speak for it (whole_is_better; never where the mean is one
  // tile: 512 requests of 1 to 32K tokens, one row of 4 heads, 343 us cut, 446
  // whole).
  s.cut = !brief && s.own_keys < keys;
  s.may_stay_whole = !one_tile;
  s.unit_log2 = 7;
  static_assert(kWaveKeys == 1 << 7, "least unit");
  // Units are counted in 32 bits.  (There are fewer than 2^27 sequences.)
  const int64_t most = int64_t{1} << 30;
  auto units_of = [&] {
    return seqs * ((keys >> s.unit_log2) + 1 + kSeqUnits);
  };
  while (units_of() >= most && s.unit_log2 < 30) ++s.unit_log2;
  s.max_units = static_cast<int>(units_of());
  const int64_t own_groups = (seqs + kWaves - 1) / kWaves;
  s.own_grid = static_cast<int>(own_groups < kOwnGrid * slots
                                    ? own_groups
                                    : kOwnGrid * slots);
  s.whole_grid = static_cast<int>(seqs < 65536 ? seqs : 65536);
  s.cut_grid = slots;
  return s;
}

// Workspace of a cut launch of `groups` workgroups: two CacheFold of each, then two
// CacheFoldKeys, then the partial results: O, reference and sum of two tiles each.
size_t fold_bytes(int groups) {
  return 2 * (sizeof(CacheFold) + sizeof(CacheFoldKeys)) * groups;
}
size_t part_rows(int groups, int nq) { return size_t{32} * nq * groups; }

template <int D, int NQ, bool OUT_F32, bool RULE, bool OWN, bool FINE>
hipError_t launch_fwd(const CacheFwdParams& p, int groups, hipStream_t stream) {
  const size_t n = static_cast<size_t>(p.num_requests);
  const size_t lds =
      (n + 1) * 4 + (n <= kKeptRequests ? n * sizeof(Request<RULE>) : 0);
  const auto kernel =
      p.c.page_log2 == 4
          ? cache_fwd_kernel<D, NQ, OUT_F32, true, OWN, RULE, FINE>
          : cache_fwd_kernel<D, NQ, OUT_F32, false, OWN, RULE, FINE>;
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(groups)), dim3(NT), lds,
                     stream, p);
  return hipGetLastError();
}

template <int D, int NQ, bool OUT_F32, bool RULE, bool FINE = OUT_F32>
hipError_t launch(CacheFwdParams p, const Shape& s, hipStream_t stream) {
  hipError_t e = hipSuccess;
  p.split = 0;
  p.least_keys = 0;
  p.most_keys = INT32_MAX;
  if (s.own_keys >= 0) {
    if (s.cut) p.most_keys = s.own_keys;
    e = launch_fwd<D, NQ, OUT_F32, RULE, true, FINE>(p, s.own_grid, stream);
    if (e != hipSuccess || !s.cut) return e;
    p.least_keys = s.own_keys + 1;
    p.most_keys = INT32_MAX;
  }
  if (!s.cut)
    return launch_fwd<D, NQ, OUT_F32, RULE, false, FINE>(p, s.whole_grid, stream);
  p.split = 1;
  e = launch_fwd<D, NQ, OUT_F32, RULE, false, FINE>(p, s.cut_grid, stream);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((cache_fold_kernel<D, NQ, OUT_F32, RULE>),
                     dim3(static_cast<unsigned>(s.cut_grid)),
                     dim3(kFoldThreads), 0, stream, p);
  return hipGetLastError();
}

template <int D, bool RULE>
hipError_t launch_d(const CacheFwdParams& p, const Shape& s, bool out_f32,
                    hipStream_t stream) {
  if constexpr (RULE) {
    if (p.wide_cap && !out_f32) {
      if constexpr (D == 64) {
        if (s.nq == 4) return launch<D, 4, false, true, true>(p, s, stream);
      }
      return s.nq == 2 ? launch<D, 2, false, true, true>(p, s, stream)
                       : launch<D, 1, false, true, true>(p, s, stream);
    }
  }
  if constexpr (!RULE || D == 64) {
    if (s.nq == 4) return launch<D, 4, false, RULE>(p, s, stream);
  }
  if (s.nq == 2)
    return out_f32 ? launch<D, 2, true, RULE>(p, s, stream)
                   : launch<D, 2, false, RULE>(p, s, stream);
  return out_f32 ? launch<D, 1, true, RULE>(p, s, stream)
                 : launch<D, 1, false, RULE>(p, s, stream);
}

}  // namespace

size_t cache_fwd_workspace(const CacheDims& c, int32_t num_requests,
                           int64_t rows) {
  if (rows == 0 || num_requests == 0 || keys_of(c) <= kBriefKeys) return 0;
  // What any call over this cache needs, so that it serves smaller ones.
  size_t most = 0;
  for (int nq = 1; nq <= 4; nq *= 2) {
    const int groups = resident_groups(c.d, nq);
    const size_t n = fold_bytes(groups) +
                     part_rows(groups, nq) * (c.d + 2) * sizeof(float);
    most = n > most ? n : most;
  }
  return most;
}

hipError_t launch_cache_fwd(const CacheFwdParams& params, bool out_f32, void* ws,
                            hipStream_t stream) {
  const Shape s = shape_of(params.c, params.hq, params.num_requests,
                           params.rows, out_f32, params.rule);
  CacheFwdParams p = params;
  p.unit_log2 = s.unit_log2;
  p.seq_units = kSeqUnits;
  p.may_stay_whole = s.may_stay_whole;
  p.max_units = s.max_units;
  int log2 = 0;
  while ((1 << log2) < p.group) ++log2;
  p.group_shift = 30 + log2;
  p.group_mul = static_cast<uint32_t>(
      ((uint64_t{1} << p.group_shift) + p.group - 1) / p.group);
  p.fold = nullptr;
  p.fold_keys = nullptr;
  p.part_o = p.part_ml = nullptr;
  if (s.cut) {
    p.fold = static_cast<CacheFold*>(ws);
    p.fold_keys = reinterpret_cast<CacheFoldKeys*>(p.fold + 2 * s.cut_grid);
    p.part_o = reinterpret_cast<float*>(static_cast<char*>(ws) +
                                        fold_bytes(s.cut_grid));
    p.part_ml = p.part_o + part_rows(s.cut_grid, s.nq) * p.c.d;
  }
  if (p.rule)
    return p.c.d == 128 ? launch_d<128, true>(p, s, out_f32, stream)
                        : launch_d<64, true>(p, s, out_f32, stream);
  return p.c.d == 128 ? launch_d<128, false>(p, s, out_f32, stream)
                      : launch_d<64, false>(p, s, out_f32, stream);
}

}  // namespace mesh_attn
