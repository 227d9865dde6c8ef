// Host side of the 4-bit key/value cache and of rotary positions: argument
// validation and launches.  Nothing here keeps state or allocates, and every
// device array is passed on unread, so the calls may be captured into graphs.

#include "cache.h"

#include <cmath>
#include <cstdint>

#include "host_error.h"
#include "mesh_attn.h"

using namespace mesh_attn;
using mesh_attn::host::fail;
using mesh_attn::host::ok;

namespace {

// A pointer argument: its name, and the alignment its kernel relies on.
struct Arg {
  const char* name;
  const void* p;
  unsigned align;
};

ma_status_t check_args(const Arg* a, int n) {
  for (int i = 0; i < n; ++i) {
    if (!a[i].p) return fail(MA_ERR_INVALID_ARG, "%s is NULL", a[i].name);
    if (reinterpret_cast<uintptr_t>(a[i].p) % a[i].align != 0)
      return fail(MA_ERR_INVALID_ARG, "%s is not %u-byte aligned", a[i].name,
                  a[i].align);
  }
  return MA_OK;
}

struct Range {
  const void* p;
  size_t bytes;
};

bool overlap(const Range& a, const Range& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p);
  const uintptr_t y = reinterpret_cast<uintptr_t>(b.p);
  return a.bytes > 0 && b.bytes > 0 && x < y + b.bytes && y < x + a.bytes;
}

ma_status_t launched(hipError_t e, const char* what) {
  if (e != hipSuccess)
    return fail(MA_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return ok();
}

ma_status_t check_cache(const ma_cache_t* c, CacheDims* out) {
  if (!c) return fail(MA_ERR_INVALID_ARG, "cache is NULL");
  if (c->num_pages < 1)
    return fail(MA_ERR_INVALID_ARG, "num_pages %d < 1", c->num_pages);
  if (c->num_kv_heads < 1 || c->num_kv_heads > 1024)
    return fail(MA_ERR_INVALID_ARG, "num_kv_heads %d outside [1, 1024]",
                c->num_kv_heads);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(MA_ERR_UNSUPPORTED, "head_dim %d: only 64 and 128",
                c->head_dim);
  int log2 = 4;
  while (log2 < 8 && (1 << log2) != c->page_size) ++log2;
  if ((1 << log2) != c->page_size)
    return fail(MA_ERR_UNSUPPORTED,
                "page_size %d: only 16, 32, 64, 128 and 256", c->page_size);
  if (c->max_pages < 1 ||
      (int64_t{c->max_pages} << log2) > (int64_t{1} << 30))
    return fail(MA_ERR_INVALID_ARG,
                "max_pages %d outside [1, 2^30 / page_size]", c->max_pages);
  if (c->layout != MA_LAYOUT_CONTIGUOUS && c->layout != MA_LAYOUT_STRIPED)
    return fail(MA_ERR_INVALID_ARG, "layout %d invalid", c->layout);
  if (c->num_partitions < 1 || c->partition < 0 ||
      c->partition >= c->num_partitions)
    return fail(MA_ERR_INVALID_ARG, "partition %d of %d invalid", c->partition,
                c->num_partitions);
  const bool striped = c->layout == MA_LAYOUT_STRIPED;
  if (!striped && c->partition_len < 1)
    return fail(MA_ERR_INVALID_ARG, "partition_len %d < 1", c->partition_len);
  out->share.striped = striped;
  out->share.n = c->num_partitions;
  out->share.p = c->partition;
  out->share.len = striped ? 0 : c->partition_len;
  out->share.first = striped ? 0 : int64_t{c->partition} * c->partition_len;
  out->num_pages = c->num_pages;
  out->page_log2 = log2;
  out->hkv = c->num_kv_heads;
  out->d = c->head_dim;
  out->max_pages = c->max_pages;
  return MA_OK;
}

constexpr int64_t kMaxRows = int64_t{1} << 31;

ma_status_t check_rows(int64_t rows) {
  if (rows < 0 || rows >= kMaxRows)
    return fail(MA_ERR_INVALID_ARG, "rows %lld outside [0, 2^31)",
                static_cast<long long>(rows));
  return MA_OK;
}

ma_status_t check_requests(int32_t n) {
  if (n < 0 || n > MA_CACHE_MAX_REQUESTS)
    return fail(MA_ERR_INVALID_ARG, "num_requests %d outside [0, %d]", n,
                MA_CACHE_MAX_REQUESTS);
  return MA_OK;
}

// A row stride in elements of which `unit` make 16 bytes.
ma_status_t check_stride(const char* name, int64_t stride, int64_t least,
                         int unit) {
  if (stride < least || stride % unit != 0 || stride > (int64_t{1} << 40))
    return fail(MA_ERR_INVALID_ARG,
                "%s %lld: need a multiple of %d, at least %lld", name,
                static_cast<long long>(stride), unit,
                static_cast<long long>(least));
  return MA_OK;
}

ma_status_t check_q_heads(int32_t hq, int32_t hkv) {
  if (hq < 1 || hq % hkv != 0 || hq > 65535)
    return fail(MA_ERR_INVALID_ARG,
                "num_q_heads %d: need a multiple of num_kv_heads %d, at most "
                "65535", hq, hkv);
  return MA_OK;
}

// f / (2 pi) modulo 1 in units of 2^-64, rounded to nearest, for |f| < 2^31: the
// kernel's product with the position wraps as turns do, so what is rounded off
// here is all that a far position's angle lacks.  f's 53-bit integer m times
// 1 / (2 pi) cut to 128 bits, of which at most 2^31 2^-128 is missing.
uint64_t turn_per_position(double f) {
  constexpr uint64_t kHigh = 0x28be60db9391054aull;
  constexpr uint64_t kLow = 0x7f09d5f47d4d3770ull;
  int exponent;
  const double fraction = std::frexp(std::fabs(f), &exponent);
  if (fraction == 0.0) return 0;
  const uint64_t m = static_cast<uint64_t>(fraction * 0x1p53);
  typedef unsigned __int128 u128;
  const u128 product = u128{kHigh} * m + ((u128{kLow} * m) >> 64);
  // The result is product 2^(exponent - 53); exponent is at most 31.
  const int shift = 52 - exponent;
  const u128 twice = shift < 128 ? product >> shift : u128{0};
  const uint64_t turn = static_cast<uint64_t>((twice + 1) >> 1);
  return f < 0 ? uint64_t{0} - turn : turn;
}

#define MA_TRY(expr)                       \
  do {                                     \
    const ma_status_t st_ = (expr);        \
    if (st_ != MA_OK) return st_;          \
  } while (0)

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
  return launched(launch_cache_fwd(p, o_dtype == MA_FP32, ws, stream),
                  "cache_fwd launch");
}

ma_status_t mesh_attn_rope(const ma_rope_t* rope, int64_t rows,
                           const int32_t* positions, int32_t q_heads,
                           const void* q, int64_t q_stride, void* q_out,
                           int64_t q_out_stride, int32_t k_heads,
                           const void* k, int64_t k_stride, void* k_out,
                           int64_t k_out_stride, ma_dtype_t dtype,
                           int32_t inverse, hipStream_t stream) {
  if (!rope) return fail(MA_ERR_INVALID_ARG, "rope is NULL");
  const int32_t d = rope->head_dim, rot = rope->rotary_dim;
  if (d < 16 || d > 256 || d % 16 != 0)
    return fail(MA_ERR_UNSUPPORTED, "head_dim %d: need a multiple of 16 in "
                "[16, 256]", d);
  if (rot < 16 || rot > d || rot % 16 != 0)
    return fail(MA_ERR_UNSUPPORTED, "rotary_dim %d: need a multiple of 16 in "
                "[16, head_dim]", rot);
  if (rope->num_axes < 1 || rope->num_axes > 8)
    return fail(MA_ERR_INVALID_ARG, "num_axes %d outside [1, 8]",
                rope->num_axes);
  if ((rope->interleaved != 0 && rope->interleaved != 1) ||
      (inverse != 0 && inverse != 1))
    return fail(MA_ERR_INVALID_ARG, "interleaved and inverse must be 0 or 1");
  if (!rope->inv_freq) return fail(MA_ERR_INVALID_ARG, "inv_freq is NULL");
  if (!rope->axis && rope->num_axes != 1)
    return fail(MA_ERR_INVALID_ARG, "axis is NULL with %d axes",
                rope->num_axes);
  if (dtype != MA_BF16 && dtype != MA_FP32)
    return fail(MA_ERR_INVALID_ARG, "dtype %d invalid", (int)dtype);
  MA_TRY(check_rows(rows));
  RopeParams p;
  for (int i = 0; i < kRopeMaxPairs; ++i) {
    p.t.turn[i] = 0;
    p.t.axis[i] = 0;
  }
  for (int i = 0; i < rot / 2; ++i) {
    const double f = rope->inv_freq[i];
    if (!(std::fabs(f) < 2147483648.0))
      return fail(MA_ERR_INVALID_ARG, "inv_freq[%d] = %g", i, f);
    p.t.turn[i] = turn_per_position(f);
    const int32_t a = rope->axis ? rope->axis[i] : 0;
    if (a < 0 || a >= rope->num_axes)
      return fail(MA_ERR_INVALID_ARG, "axis[%d] = %d outside [0, %d)", i, a,
                  rope->num_axes);
    p.t.axis[i] = static_cast<uint8_t>(a);
  }
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
