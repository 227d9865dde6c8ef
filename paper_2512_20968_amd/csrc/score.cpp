// Host side of the attention under a score rule over a tile: argument validation,
// the KV buffer's segments, workspaces and launches.  Nothing here keeps state or
// allocates, and every device array is passed on unread, so the calls may be
// captured into graphs.

#include "score.h"

#include <cmath>
#include <cstdint>

#include "cache_args.h"
#include "mesh_attn.h"

using namespace mesh_attn;
using namespace mesh_attn::host;

namespace {

constexpr float kLog2e = 1.4426950408889634f;

ma_status_t check_score_problem(const ma_problem_t* prob, int32_t nq,
                                int32_t nkv) {
  MA_TRY(check_problem(prob));
  if (prob->head_dim != 64 && prob->head_dim != 128)
    return fail(MA_ERR_UNSUPPORTED, "head_dim %d unsupported (64 or 128)",
                prob->head_dim);
  if (!std::isfinite(prob->softmax_scale * kLog2e))
    return fail(MA_ERR_INVALID_ARG, "softmax_scale %g is too large",
                prob->softmax_scale);
  if (nq < 1 || nkv < 1 || nq > kScoreMaxList || nkv > kScoreMaxList)
    return fail(nq < 1 || nkv < 1 ? MA_ERR_INVALID_ARG : MA_ERR_UNSUPPORTED,
                "lists of %d and %d partitions: need 1 to %d", nq, nkv,
                kScoreMaxList);
  if (prob->num_q_heads > 65535)
    return fail(MA_ERR_UNSUPPORTED, "num_q_heads %d above 65535",
                prob->num_q_heads);
  // The backward's first launch has d / 8 lanes for every head of every row, in
  // stages of 64, counted in 32 bits.
  const int64_t most = int64_t{1} << 27;
  const int64_t q = int64_t{nq} * prob->partition_len + 63;
  const int64_t kv = int64_t{nkv} * prob->partition_len + 63;
  if (nq > prob->num_partitions || nkv > prob->num_partitions)
    return fail(MA_ERR_INVALID_ARG, "lists of %d and %d partitions of %d", nq,
                nkv, prob->num_partitions);
  if (q > most / prob->num_q_heads || kv > most / prob->num_kv_heads)
    return fail(MA_ERR_UNSUPPORTED, "rows times heads above 2^27");
  return MA_OK;
}

ma_status_t check_indices(const char* name, const int32_t* idx, int32_t n,
                          int32_t num_partitions) {
  if (!idx) return fail(MA_ERR_INVALID_ARG, "%s is NULL", name);
  for (int32_t i = 0; i < n; ++i) {
    if (idx[i] < 0 || idx[i] >= num_partitions)
      return fail(MA_ERR_INVALID_ARG, "%s[%d] = %d outside [0, %d)", name, i,
                  idx[i], num_partitions);
    for (int32_t j = 0; j < i; ++j)
      if (idx[i] == idx[j])
        return fail(MA_ERR_INVALID_ARG, "%s[%d] = %d is a duplicate", name, i,
                    idx[i]);
  }
  return MA_OK;
}

// Row strides below this keep a stage of 64 rows within 32 bits.
constexpr int64_t kMaxStride = int64_t{1} << 24;

ma_status_t check_row_stride(const char* name, int64_t stride, int64_t least) {
  MA_TRY(check_stride(name, stride, least, 8));
  if (stride > kMaxStride)
    return fail(MA_ERR_UNSUPPORTED, "%s %lld above 2^24", name,
                static_cast<long long>(stride));
  return MA_OK;
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Sizes of a tile, as far as they are known without its lists.
void fill_sizes(const ma_problem_t& p, int32_t nq, int32_t nkv, ScoreTile* t) {
  t->rows_q = nq * p.partition_len;
  t->rows_kv = nkv * p.partition_len;
  t->hq = p.num_q_heads;
  t->hkv = p.num_kv_heads;
  t->group = p.num_q_heads / p.num_kv_heads;
  t->head_dim = p.head_dim;
  t->P = p.partition_len;
  t->n = p.num_partitions;
  t->striped = p.layout == MA_LAYOUT_STRIPED;
  t->step = t->striped ? p.num_partitions : 1;
  t->causal = p.causal;
  t->total = p.num_partitions * p.partition_len;
  t->scale = p.softmax_scale;
  t->scale_log2 = p.softmax_scale * kLog2e;
  // Most blocks: no segment merged.
  t->kv_blocks64 = nkv * ((t->P + 63) / 64);
  t->kv_blocks128 = nkv * ((t->P + 127) / 128);
}

void fill_segments(const int32_t* q_idx, int32_t nq, const int32_t* kv_idx,
                   int32_t nkv, ScoreTile* t) {
  for (int i = 0; i < nq; ++i) t->q_idx[i] = q_idx[i];
  t->nseg = 0;
  for (int i = 0; i < nkv; ++i) {
    if (!t->striped && i > 0 && kv_idx[i] == kv_idx[i - 1] + 1) continue;
    t->seg_row[t->nseg] = i * t->P;
    t->seg_pos[t->nseg] = t->striped ? kv_idx[i] : kv_idx[i] * t->P;
    ++t->nseg;
  }
  t->seg_row[t->nseg] = t->rows_kv;
  t->kv_blocks64 = t->kv_blocks128 = 0;
  for (int s = 0; s < t->nseg; ++s) {
    const int len = t->seg_row[s + 1] - t->seg_row[s];
    t->kv_blocks64 += (len + 63) / 64;
    t->kv_blocks128 += (len + 127) / 128;
  }
}

ma_status_t check_tile(const ma_problem_t* prob, const int32_t* q_idx,
                       int32_t nq, const int32_t* kv_idx, int32_t nkv,
                       const ma_score_t* score, const void* q,
                       int64_t q_stride, const void* k, int64_t k_stride,
                       const void* v, int64_t v_stride, ScoreTile* t) {
  MA_TRY(check_score_problem(prob, nq, nkv));
  MA_TRY(check_indices("q_idx", q_idx, nq, prob->num_partitions));
  MA_TRY(check_indices("kv_idx", kv_idx, nkv, prob->num_partitions));
  MA_TRY(check_score(score, prob->softmax_scale));
  // The kernels take the distances within a block of 64 keys in float32.
  if (score && score->slopes && prob->layout == MA_LAYOUT_STRIPED &&
      prob->num_partitions > 1 << 18)
    return fail(MA_ERR_UNSUPPORTED,
                "slopes with %d striped partitions, above 2^18",
                prob->num_partitions);
  const int64_t d = prob->head_dim;
  MA_TRY(check_row_stride("q_stride", q_stride, prob->num_q_heads * d));
  MA_TRY(check_row_stride("k_stride", k_stride, prob->num_kv_heads * d));
  MA_TRY(check_row_stride("v_stride", v_stride, prob->num_kv_heads * d));
  const Arg args[] = {{"q", q, 16}, {"k", k, 16}, {"v", v, 16}};
  MA_TRY(check_args(args, 3));
  fill_sizes(*prob, nq, nkv, t);
  fill_segments(q_idx, nq, kv_idx, nkv, t);
  t->q = static_cast<const uint16_t*>(q);
  t->k = static_cast<const uint16_t*>(k);
  t->v = static_cast<const uint16_t*>(v);
  t->q_stride = q_stride;
  t->k_stride = k_stride;
  t->v_stride = v_stride;
  t->cap = score ? score->cap : 0.f;
  t->slopes = score ? score->slopes : nullptr;
  t->key_begin = score ? score->key_begin : nullptr;
  t->key_end = score ? score->key_end : nullptr;
  return MA_OK;
}

// The buffers that a call reads, for the check that no output lies in them.
int inputs_of(const ScoreTile& t, Range* r) {
  const size_t rq = static_cast<size_t>(t.rows_q);
  const size_t rk = static_cast<size_t>(t.rows_kv);
  const auto strided = [&](size_t rows, int64_t stride, int heads) {
    return 2 * ((rows - 1) * static_cast<size_t>(stride) +
                static_cast<size_t>(heads) * static_cast<size_t>(t.head_dim));
  };
  r[0] = {t.q, strided(rq, t.q_stride, t.hq)};
  r[1] = {t.k, strided(rk, t.k_stride, t.hkv)};
  r[2] = {t.v, strided(rk, t.v_stride, t.hkv)};
  r[3] = {t.slopes, t.slopes ? 4 * static_cast<size_t>(t.hq) : 0};
  r[4] = {t.key_begin, t.key_begin ? 4 * rq : 0};
  r[5] = {t.key_end, t.key_end ? 4 * rq : 0};
  return 6;
}

// ranges: `outputs` outputs, then inputs.
ma_status_t check_apart(const Range* ranges, int outputs, int n) {
  for (int i = 0; i < outputs; ++i)
    for (int j = i + 1; j < n; ++j)
      if (overlap(ranges[i], ranges[j]))
        return fail(MA_ERR_INVALID_ARG,
                    "an output must not alias an input or another output");
  return MA_OK;
}

size_t fwd_bytes(const ScoreTile& t, int splits) {
  if (splits == 1) return 0;
  const size_t items = static_cast<size_t>(t.rows_q) * t.hq * splits;
  return up256(4 * items * t.head_dim) + up256(4 * items);
}

struct BwdBytes {
  size_t rows, ints, stages, counts, kv, q, all;
};

BwdBytes bwd_bytes(const ScoreTile& t, int kv_splits, int q_splits) {
  const size_t pad = (static_cast<size_t>(t.rows_q) + 63) / 64 * 64;
  BwdBytes b;
  b.rows = up256(4 * pad * t.hq);
  b.ints = up256(4 * pad);
  b.stages = up256(sizeof(ScoreStage) * (pad / 64));
  b.counts = kv_splits == 1
                 ? 0
                 : up256(4 * static_cast<size_t>(t.rows_kv) * t.hkv);
  b.kv = kv_splits == 1 ? 0
                        : up256(4 * static_cast<size_t>(t.rows_kv) * t.hkv *
                                t.head_dim * kv_splits);
  b.q = q_splits == 1 ? 0
                      : up256(4 * static_cast<size_t>(t.rows_q) * t.hq *
                              t.head_dim * q_splits);
  b.all = 2 * b.rows + 4 * b.ints + b.stages + b.counts +
          2 * b.kv + b.q;
  return b;
}

}  // namespace

extern "C" {

size_t mesh_attn_score_fwd_workspace_size(const ma_problem_t* prob, int32_t nq,
                                          int32_t nkv) {
  if (check_score_problem(prob, nq, nkv) != MA_OK) return 0;
  ok();
  ScoreTile t;
  fill_sizes(*prob, nq, nkv, &t);
  return fwd_bytes(t, score_fwd_splits(t));
}

ma_status_t mesh_attn_score_fwd(const ma_problem_t* prob, const int32_t* q_idx,
                                int32_t nq, const int32_t* kv_idx, int32_t nkv,
                                const ma_score_t* score, const void* q,
                                int64_t q_stride, const void* k,
                                int64_t k_stride, const void* v,
                                int64_t v_stride, void* o, ma_dtype_t o_dtype,
                                float* lse, void* ws, size_t ws_bytes,
                                hipStream_t stream) {
  ScoreFwdParams p;
  MA_TRY(check_tile(prob, q_idx, nq, kv_idx, nkv, score, q, q_stride, k,
                    k_stride, v, v_stride, &p.t));
  if (o_dtype != MA_BF16 && o_dtype != MA_FP32)
    return fail(MA_ERR_INVALID_ARG, "o_dtype %d invalid", (int)o_dtype);
  const Arg args[] = {{"o", o, 16}, {"lse", lse, 16}};
  MA_TRY(check_args(args, 2));
  p.splits = score_fwd_splits(p.t);
  const size_t need = fwd_bytes(p.t, p.splits);
  if (need > 0) {
    if (ws_bytes < need)
      return fail(MA_ERR_WORKSPACE_TOO_SMALL,
                  "workspace of %zu bytes, %zu needed", ws_bytes, need);
    const Arg a{"ws", ws, 16};
    MA_TRY(check_args(&a, 1));
  }
  const size_t values = static_cast<size_t>(p.t.rows_q) * p.t.hq;
  Range r[9] = {{o, values * p.t.head_dim * (o_dtype == MA_FP32 ? 4 : 2)},
                {lse, 4 * values},
                {ws, need}};
  MA_TRY(check_apart(r, 3, 3 + inputs_of(p.t, r + 3)));
  p.o = o;
  p.lse = lse;
  p.part_o = static_cast<float*>(ws);
  p.part_lse =
      need == 0 ? nullptr
                : reinterpret_cast<float*>(
                      static_cast<char*>(ws) +
                      up256(4 * values * p.t.head_dim * p.splits));
  return launched(launch_score_fwd(p, o_dtype == MA_FP32, stream),
                  "score_fwd launch");
}

size_t mesh_attn_score_bwd_workspace_size(const ma_problem_t* prob, int32_t nq,
                                          int32_t nkv) {
  if (check_score_problem(prob, nq, nkv) != MA_OK) return 0;
  ok();
  ScoreTile t;
  fill_sizes(*prob, nq, nkv, &t);
  // Most parts: the fewest blocks of 128 keys (all segments merged), the most of
  // 64.
  t.kv_blocks128 = (t.rows_kv + 127) / 128;
  int kv, qs;
  score_bwd_splits(t, &kv, &qs);
  return bwd_bytes(t, kv, qs).all;
}

ma_status_t mesh_attn_score_bwd(const ma_problem_t* prob, const int32_t* q_idx,
                                int32_t nq, const int32_t* kv_idx, int32_t nkv,
                                const ma_score_t* score, const void* q,
                                int64_t q_stride, const void* k,
                                int64_t k_stride, const void* v,
                                int64_t v_stride, const void* o,
                                const void* d_o, const float* lse, void* dq,
                                void* dk, void* dv, ma_dtype_t grad_dtype,
                                void* ws, size_t ws_bytes,
                                hipStream_t stream) {
  ScoreBwdParams p;
  MA_TRY(check_tile(prob, q_idx, nq, kv_idx, nkv, score, q, q_stride, k,
                    k_stride, v, v_stride, &p.t));
  if (grad_dtype != MA_BF16 && grad_dtype != MA_FP32)
    return fail(MA_ERR_INVALID_ARG, "grad_dtype %d invalid", (int)grad_dtype);
  const Arg args[] = {{"o", o, 16},   {"d_o", d_o, 16}, {"lse", lse, 16},
                      {"dq", dq, 16}, {"dk", dk, 16},   {"dv", dv, 16},
                      {"ws", ws, 16}};
  MA_TRY(check_args(args, 7));
  score_bwd_splits(p.t, &p.kv_splits, &p.q_splits);
  const BwdBytes b = bwd_bytes(p.t, p.kv_splits, p.q_splits);
  if (ws_bytes < b.all)
    return fail(MA_ERR_WORKSPACE_TOO_SMALL,
                "workspace of %zu bytes, %zu needed", ws_bytes, b.all);
  const size_t rq = static_cast<size_t>(p.t.rows_q) * p.t.hq;
  const size_t rk = static_cast<size_t>(p.t.rows_kv) * p.t.hkv;
  const size_t d = static_cast<size_t>(p.t.head_dim);
  const size_t g = grad_dtype == MA_FP32 ? 4 : 2;
  Range r[13] = {{dq, rq * d * g}, {dk, rk * d * g}, {dv, rk * d * g},
                 {ws, b.all},      {o, rq * d * 2},  {d_o, rq * d * 2},
                 {lse, 4 * rq}};
  MA_TRY(check_apart(r, 4, 7 + inputs_of(p.t, r + 7)));
  p.o = static_cast<const uint16_t*>(o);
  p.d_o = static_cast<const uint16_t*>(d_o);
  p.lse = lse;
  p.dq = dq;
  p.dk = dk;
  p.dv = dv;
  p.rows_pad = (p.t.rows_q + 63) / 64 * 64;
  char* at = static_cast<char*>(ws);
  const auto take = [&](size_t bytes) {
    char* x = at;
    at += bytes;
    return x;
  };
  p.delta = reinterpret_cast<float*>(take(b.rows));
  p.lse2 = reinterpret_cast<float*>(take(b.rows));
  p.lo = reinterpret_cast<int32_t*>(take(b.ints));
  p.hi = reinterpret_cast<int32_t*>(take(b.ints));
  p.pos = reinterpret_cast<int32_t*>(take(b.ints));
  p.pos_rel = reinterpret_cast<float*>(take(b.ints));
  p.stages = reinterpret_cast<ScoreStage*>(take(b.stages));
  p.kv_parts = reinterpret_cast<int32_t*>(take(b.counts));
  p.part_dk = reinterpret_cast<float*>(take(b.kv));
  p.part_dv = reinterpret_cast<float*>(take(b.kv));
  p.part_dq = reinterpret_cast<float*>(take(b.q));
  return launched(launch_score_bwd(p, grad_dtype == MA_FP32, stream),
                  "score_bwd launch");
}

ma_status_t mesh_attn_cache_rope_append(
    const ma_cache_t* cache, const ma_rope_t* rope, int64_t rows,
    const int32_t* positions, int32_t q_heads, const void* q, int64_t q_stride,
    void* q_out, int64_t q_out_stride, const void* k, int64_t k_stride,
    const void* v, int64_t v_stride, const int64_t* slots, void* data,
    hipStream_t stream) {
  RopeAppendParams p;
  MA_TRY(check_cache(cache, &p.c));
  MA_TRY(check_rope(rope, &p.t));
  if (rope->head_dim != p.c.d)
    return fail(MA_ERR_INVALID_ARG, "head_dim %d of the rotation, %d of the "
                "cache", rope->head_dim, p.c.d);
  MA_TRY(check_rows(rows));
  if (q_heads < 1 || q_heads > 65535)
    return fail(MA_ERR_INVALID_ARG, "q_heads %d outside [1, 65535]", q_heads);
  const int64_t qw = int64_t{q_heads} * p.c.d, kw = int64_t{p.c.hkv} * p.c.d;
  MA_TRY(check_stride("q_stride", q_stride, qw, 8));
  MA_TRY(check_stride("q_out_stride", q_out_stride, qw, 8));
  MA_TRY(check_stride("k_stride", k_stride, kw, 8));
  MA_TRY(check_stride("v_stride", v_stride, kw, 8));
  if (q == q_out && q_stride != q_out_stride)
    return fail(MA_ERR_INVALID_ARG, "in place with different strides");
  if (rows == 0) return ok();
  const Arg args[] = {{"positions", positions, 4}, {"q", q, 16},
                      {"q_out", q_out, 16},        {"k", k, 16},
                      {"v", v, 16},                {"slots", slots, 8},
                      {"data", data, 16}};
  MA_TRY(check_args(args, 7));
  p.positions = positions;
  p.q = static_cast<const uint16_t*>(q);
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.q_out = static_cast<uint16_t*>(q_out);
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.q_out_stride = q_out_stride;
  p.slots = slots;
  p.data = static_cast<uint8_t*>(data);
  p.rows = rows;
  p.hq = q_heads;
  p.rot = rope->rotary_dim;
  p.interleaved = rope->interleaved;
  return launched(launch_rope_append(p, stream), "rope_append launch");
}

}  // extern "C"
