// Host side of the 4-bit key/value cache and of rotary positions: argument
// validation and launches.  Nothing here keeps state or allocates, and every
// device array is passed on unread, so the calls may be captured into graphs.

#include "cache.h"

#include <cmath>
#include <cstdint>

#include "cache_args.h"
#include "mesh_attn.h"

using namespace mesh_attn;
using namespace mesh_attn::host;

namespace {

// Attention over the cache, with a score rule or without.
ma_status_t cache_fwd(
    const ma_cache_t* cache, int32_t num_q_heads, float softmax_scale,
    bool rule, const ma_score_t* score, int32_t num_requests, int64_t rows,
    const void* q, int64_t q_stride, const int32_t* positions,
    const int32_t* cu_new, const int32_t* lens, const int32_t* block_table,
    const void* data, void* o, ma_dtype_t o_dtype, float* lse, void* ws,
    size_t ws_bytes, hipStream_t stream) {
  CacheFwdParams p;
  MA_TRY(check_cache(cache, &p.c));
  MA_TRY(check_q_heads(num_q_heads, p.c.hkv));
  MA_TRY(check_requests(num_requests));
  MA_TRY(check_rows(rows));
  p.scale_log2 = softmax_scale * 1.4426950408889634f;
  p.inv_scale_log2 = 1.f / p.scale_log2;
  if (!(softmax_scale > 0.f) || !std::isfinite(p.scale_log2))
    return fail(MA_ERR_INVALID_ARG, "softmax_scale must be positive and "
                "finite");
  if (rule) MA_TRY(check_score(score, softmax_scale));
  if (o_dtype != MA_BF16 && o_dtype != MA_FP32)
    return fail(MA_ERR_INVALID_ARG, "o_dtype %d invalid", (int)o_dtype);
  if (rows * num_q_heads >= int64_t{1} << 30)
    return fail(MA_ERR_INVALID_ARG, "rows * num_q_heads %lld not below 2^30",
                static_cast<long long>(rows) * num_q_heads);
  MA_TRY(check_stride("q_stride", q_stride, int64_t{num_q_heads} * p.c.d, 8));
  if (rows == 0 || num_requests == 0) return ok();
  const Arg args[] = {{"q", q, 16},
                      {"positions", positions, 4},
                      {"cu_new", cu_new, 4},
                      {"lens", lens, 4},
                      {"block_table", block_table, 4},
                      {"data", data, 16},
                      {"o", o, 16},
                      {"lse", lse, 4}};
  MA_TRY(check_args(args, 8));
  const size_t need = cache_fwd_workspace(p.c, num_requests, rows);
  if (need > 0) {
    if (ws_bytes < need)
      return fail(MA_ERR_WORKSPACE_TOO_SMALL,
                  "workspace of %zu bytes, %zu needed", ws_bytes, need);
    const Arg a{"ws", ws, 16};
    MA_TRY(check_args(&a, 1));
  }
  p.q = static_cast<const uint16_t*>(q);
  p.q_stride = q_stride;
  p.positions = positions;
  p.cu = cu_new;
  p.lens = lens;
  p.block_table = block_table;
  p.data = static_cast<const uint8_t*>(data);
  p.o = o;
  p.lse = lse;
  p.rows = rows;
  p.hq = num_q_heads;
  p.group = num_q_heads / p.c.hkv;
  p.num_requests = num_requests;
  p.rule = rule;
  p.wide_cap = score && score->cap > kWideCap;
  p.cap_in = p.cap_two = p.cap_u = 0.f;
  p.slopes = nullptr;
  p.key_begin = p.key_end = nullptr;
  if (score) {
    if (score->cap > 0.f) {
      p.cap_in = 2.f * p.scale_log2 / score->cap;
      p.cap_two = 2.f * score->cap * 1.4426950408889634f;
      p.cap_u = softmax_scale / score->cap;
    }
    p.slopes = score->slopes;
    p.key_begin = score->key_begin;
    p.key_end = score->key_end;
  }
  return launched(launch_cache_fwd(p, o_dtype == MA_FP32, ws, stream),
                  "cache_fwd launch");
}

}  // namespace

extern "C" {

size_t mesh_attn_cache_bytes(const ma_cache_t* cache) {
  CacheDims c;
  if (check_cache(cache, &c) != MA_OK) return 0;
  ok();
  return static_cast<size_t>(c.num_pages) * static_cast<size_t>(c.hkv) *
         static_cast<size_t>(c.block_bytes());
}

ma_status_t mesh_attn_cache_tables(
    const ma_cache_t* cache, int32_t num_requests, const int32_t* lens,
    const int32_t* new_lens, const int32_t* free_pages, int32_t num_free,
    const int32_t* free_range, int32_t* block_table, int32_t* lens_out,
    int32_t* cu_new, int64_t rows, int64_t* slots, int32_t* positions,
    int32_t* free_range_out, int32_t* refused, hipStream_t stream) {
  TablesParams p;
  MA_TRY(check_cache(cache, &p.c));
  MA_TRY(check_requests(num_requests));
  MA_TRY(check_rows(rows));
  if (num_free < 0)
    return fail(MA_ERR_INVALID_ARG, "num_free %d < 0", num_free);
  const Arg always[] = {{"free_range", free_range, 4},
                        {"cu_new", cu_new, 4},
                        {"free_range_out", free_range_out, 4},
                        {"refused", refused, 4}};
  MA_TRY(check_args(always, 4));
  if (num_requests > 0) {
    const Arg args[] = {{"lens", lens, 4},
                        {"new_lens", new_lens, 4},
                        {"block_table", block_table, 4},
                        {"lens_out", lens_out, 4}};
    MA_TRY(check_args(args, 4));
  }
  if (num_free > 0) {
    const Arg a{"free_pages", free_pages, 4};
    MA_TRY(check_args(&a, 1));
  }
  if (rows > 0) {
    const Arg args[] = {{"slots", slots, 8}, {"positions", positions, 4}};
    MA_TRY(check_args(args, 2));
  }
  // Outputs, then inputs: the former are written while other workgroups of the
  // launch still read the latter.
  const size_t n = static_cast<size_t>(num_requests);
  const Range ranges[] = {
      {block_table, 4 * n * static_cast<size_t>(p.c.max_pages)},
      {lens_out, 4 * n},
      {cu_new, 4 * (n + 1)},
      {slots, 8 * static_cast<size_t>(rows)},
      {positions, 4 * static_cast<size_t>(rows)},
      {free_range_out, 8},
      {refused, 4},
      {lens, 4 * n},
      {new_lens, 4 * n},
      {free_pages, 4 * static_cast<size_t>(num_free)},
      {free_range, 8}};
  constexpr int kOutputs = 7, kRanges = 11;
  for (int i = 0; i < kOutputs; ++i)
    for (int j = i + 1; j < kRanges; ++j)
      if (overlap(ranges[i], ranges[j]))
        return fail(MA_ERR_INVALID_ARG,
                    "an output must not alias an input or another output");
  p.lens = lens;
  p.new_lens = new_lens;
  p.free_pages = free_pages;
  p.free_range = free_range;
  p.block_table = block_table;
  p.lens_out = lens_out;
  p.cu_new = cu_new;
  p.slots = slots;
  p.positions = positions;
  p.free_range_out = free_range_out;
  p.refused = refused;
  p.rows = rows;
  p.num_requests = num_requests;
  p.num_free = num_free;
  return launched(launch_cache_tables(p, stream), "cache_tables launch");
}

ma_status_t mesh_attn_cache_append(const ma_cache_t* cache, int64_t rows,
                                   const void* k, int64_t k_stride,
                                   const void* v, int64_t v_stride,
                                   const int64_t* slots, void* data,
                                   hipStream_t stream) {
  StoreParams p;
  MA_TRY(check_cache(cache, &p.c));
  MA_TRY(check_rows(rows));
  const int64_t width = int64_t{p.c.hkv} * p.c.d;
  MA_TRY(check_stride("k_stride", k_stride, width, 8));
  MA_TRY(check_stride("v_stride", v_stride, width, 8));
  if (rows == 0) return ok();
  const Arg args[] = {
      {"k", k, 16}, {"v", v, 16}, {"slots", slots, 8}, {"data", data, 16}};
  MA_TRY(check_args(args, 4));
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.slots = slots;
  p.data = static_cast<uint8_t*>(data);
  p.rows = rows;
  return launched(launch_cache_append(p, stream), "cache_append launch");
}

ma_status_t mesh_attn_cache_read(const ma_cache_t* cache, int64_t rows,
                                 const int64_t* slots, const void* data,
                                 void* k, void* v, hipStream_t stream) {
  LoadParams p;
  MA_TRY(check_cache(cache, &p.c));
  MA_TRY(check_rows(rows));
  if (rows == 0) return ok();
  const Arg args[] = {
      {"slots", slots, 8}, {"data", data, 16}, {"k", k, 16}, {"v", v, 16}};
  MA_TRY(check_args(args, 4));
  p.slots = slots;
  p.data = static_cast<const uint8_t*>(data);
  p.k = static_cast<uint16_t*>(k);
  p.v = static_cast<uint16_t*>(v);
  p.rows = rows;
  return launched(launch_cache_read(p, stream), "cache_read launch");
}

size_t mesh_attn_cache_fwd_workspace_size(const ma_cache_t* cache,
                                          int32_t num_q_heads,
                                          int32_t num_requests, int64_t rows) {
  CacheDims c;
  if (check_cache(cache, &c) != MA_OK ||
      check_q_heads(num_q_heads, c.hkv) != MA_OK ||
      check_requests(num_requests) != MA_OK || check_rows(rows) != MA_OK)
    return 0;
  ok();
  return cache_fwd_workspace(c, num_requests, rows);
}

ma_status_t mesh_attn_cache_fwd(
    const ma_cache_t* cache, int32_t num_q_heads, float softmax_scale,
    int32_t num_requests, int64_t rows, const void* q, int64_t q_stride,
    const int32_t* positions, const int32_t* cu_new, const int32_t* lens,
    const int32_t* block_table, const void* data, void* o, ma_dtype_t o_dtype,
    float* lse, void* ws, size_t ws_bytes, hipStream_t stream) {
  return cache_fwd(cache, num_q_heads, softmax_scale, false, nullptr,
                   num_requests, rows, q, q_stride, positions, cu_new, lens,
                   block_table, data, o, o_dtype, lse, ws, ws_bytes, stream);
}

size_t mesh_attn_cache_score_fwd_workspace_size(const ma_cache_t* cache,
                                                int32_t num_q_heads,
                                                int32_t num_requests,
                                                int64_t rows) {
  return mesh_attn_cache_fwd_workspace_size(cache, num_q_heads, num_requests,
                                            rows);
}

ma_status_t mesh_attn_cache_score_fwd(
    const ma_cache_t* cache, int32_t num_q_heads, float softmax_scale,
    const ma_score_t* score, int32_t num_requests, int64_t rows, const void* q,
    int64_t q_stride, const int32_t* positions, const int32_t* cu_new,
    const int32_t* lens, const int32_t* block_table, const void* data, void* o,
    ma_dtype_t o_dtype, float* lse, void* ws, size_t ws_bytes,
    hipStream_t stream) {
  return cache_fwd(cache, num_q_heads, softmax_scale, true, score,
                   num_requests, rows, q, q_stride, positions, cu_new, lens,
                   block_table, data, o, o_dtype, lse, ws, ws_bytes, stream);
}

ma_status_t mesh_attn_rope(const ma_rope_t* rope, int64_t rows,
                           const int32_t* positions, int32_t q_heads,
                           const void* q, int64_t q_stride, void* q_out,
                           int64_t q_out_stride, int32_t k_heads,
                           const void* k, int64_t k_stride, void* k_out,
                           int64_t k_out_stride, ma_dtype_t dtype,
                           int32_t inverse, hipStream_t stream) {
  RopeParams p;
  if (inverse != 0 && inverse != 1)
    return fail(MA_ERR_INVALID_ARG, "interleaved and inverse must be 0 or 1");
  MA_TRY(check_rope(rope, &p.t));
  const int32_t d = rope->head_dim, rot = rope->rotary_dim;
  if (dtype != MA_BF16 && dtype != MA_FP32)
    return fail(MA_ERR_INVALID_ARG, "dtype %d invalid", (int)dtype);
  MA_TRY(check_rows(rows));
  if (q_heads < 1 || q_heads > 65535 || k_heads < 0 || k_heads > 65535)
    return fail(MA_ERR_INVALID_ARG, "q_heads %d, k_heads %d outside [1, 65535]"
                " and [0, 65535]", q_heads, k_heads);
  const int unit = dtype == MA_FP32 ? 4 : 8;
  MA_TRY(check_stride("q_stride", q_stride, int64_t{q_heads} * d, unit));
  MA_TRY(check_stride("q_out_stride", q_out_stride, int64_t{q_heads} * d,
                      unit));
  if (k_heads > 0) {
    MA_TRY(check_stride("k_stride", k_stride, int64_t{k_heads} * d, unit));
    MA_TRY(check_stride("k_out_stride", k_out_stride, int64_t{k_heads} * d,
                        unit));
  }
  if ((q == q_out && q_stride != q_out_stride) ||
      (k_heads > 0 && k == k_out && k_stride != k_out_stride))
    return fail(MA_ERR_INVALID_ARG, "in place with different strides");
  if (rows == 0) return ok();
  const Arg args[] = {{"positions", positions, 4}, {"q", q, 16},
                      {"q_out", q_out, 16},        {"k", k, 16},
                      {"k_out", k_out, 16}};
  MA_TRY(check_args(args, k_heads > 0 ? 5 : 3));
  p.positions = positions;
  p.x[0] = q;
  p.x[1] = k;
  p.y[0] = q_out;
  p.y[1] = k_out;
  p.x_stride[0] = q_stride;
  p.x_stride[1] = k_stride;
  p.y_stride[0] = q_out_stride;
  p.y_stride[1] = k_out_stride;
  p.rows = rows;
  p.heads[0] = q_heads;
  p.heads[1] = k_heads;
  p.d = d;
  p.rot = rot;
  p.interleaved = rope->interleaved;
  p.inverse = inverse;
  return launched(launch_rope(p, dtype == MA_FP32, stream), "rope launch");
}

}  // extern "C"
