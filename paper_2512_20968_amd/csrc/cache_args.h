// Checks of arguments shared by the host side of the cache, rotation and score
// calls.
#pragma once

#include <cmath>
#include <cstdint>

#include "cache.h"
#include "host_error.h"
#include "mesh_attn.h"

#define MA_TRY(expr)                       \
  do {                                     \
    const ma_status_t st_ = (expr);        \
    if (st_ != MA_OK) return st_;          \
  } while (0)

namespace mesh_attn {
namespace host {

// A pointer argument: its name, and the alignment its kernel relies on.
struct Arg {
  const char* name;
  const void* p;
  unsigned align;
};

inline ma_status_t check_args(const Arg* a, int n) {
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

inline bool overlap(const Range& a, const Range& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p);
  const uintptr_t y = reinterpret_cast<uintptr_t>(b.p);
  return a.bytes > 0 && b.bytes > 0 && x < y + b.bytes && y < x + a.bytes;
}

inline ma_status_t launched(hipError_t e, const char* what) {
  if (e != hipSuccess)
    return fail(MA_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return ok();
}

inline ma_status_t check_cache(const ma_cache_t* c, CacheDims* out) {
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

inline ma_status_t check_rows(int64_t rows) {
  if (rows < 0 || rows >= kMaxRows)
    return fail(MA_ERR_INVALID_ARG, "rows %lld outside [0, 2^31)",
                static_cast<long long>(rows));
  return MA_OK;
}

inline ma_status_t check_requests(int32_t n) {
  if (n < 0 || n > MA_CACHE_MAX_REQUESTS)
    return fail(MA_ERR_INVALID_ARG, "num_requests %d outside [0, %d]", n,
                MA_CACHE_MAX_REQUESTS);
  return MA_OK;
}

// A row stride in elements of which `unit` make 16 bytes.
inline ma_status_t check_stride(const char* name, int64_t stride, int64_t least,
                         int unit) {
  if (stride < least || stride % unit != 0 || stride > (int64_t{1} << 40))
    return fail(MA_ERR_INVALID_ARG,
                "%s %lld: need a multiple of %d, at least %lld", name,
                static_cast<long long>(stride), unit,
                static_cast<long long>(least));
  return MA_OK;
}

inline ma_status_t check_q_heads(int32_t hq, int32_t hkv) {
  if (hq < 1 || hq % hkv != 0 || hq > 65535)
    return fail(MA_ERR_INVALID_ARG,
                "num_q_heads %d: need a multiple of num_kv_heads %d, at most "
                "65535", hq, hkv);
  return MA_OK;
}

// A score rule: a cap of 0 or a positive one that the scores can be divided by.
// (Up to 2^100: a score over the cap is then a normal float32 down to scores of
// 2^-26.)
inline ma_status_t check_score(const ma_score_t* s, float softmax_scale) {
  if (!s) return MA_OK;
  if (!(s->cap >= 0.f) || !std::isfinite(s->cap))
    return fail(MA_ERR_INVALID_ARG, "cap must be 0 or positive and finite");
  if (s->cap > 0.f) {
    const float in = 2.f * softmax_scale * 1.4426950408889634f / s->cap;
    if (!std::isfinite(in) || !(in >= 0x1p-124f) || s->cap > 0x1p100f)
      return fail(MA_ERR_INVALID_ARG, "cap %g: out of range of the scores",
                  s->cap);
  }
  const Arg args[] = {{"slopes", s->slopes, 4},
                      {"key_begin", s->key_begin, 4},
                      {"key_end", s->key_end, 4}};
  for (const Arg& a : args)
    if (a.p) MA_TRY(check_args(&a, 1));
  return MA_OK;
}

// f / (2 pi) modulo 1 in units of 2^-64, rounded to nearest, for |f| < 2^31: the
// kernel's product with the position wraps as turns do, so what is rounded off
// here is all that a far position's angle lacks.  f's 53-bit integer m times
// 1 / (2 pi) cut to 128 bits, of which at most 2^31 2^-128 is missing.
inline uint64_t turn_per_position(double f) {
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

// A rotation's description; its pairs' turns and axes into *t.
inline ma_status_t check_rope(const ma_rope_t* rope, RopeTable* t) {
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
  if (rope->interleaved != 0 && rope->interleaved != 1)
    return fail(MA_ERR_INVALID_ARG, "interleaved and inverse must be 0 or 1");
  if (!rope->inv_freq) return fail(MA_ERR_INVALID_ARG, "inv_freq is NULL");
  if (!rope->axis && rope->num_axes != 1)
    return fail(MA_ERR_INVALID_ARG, "axis is NULL with %d axes",
                rope->num_axes);
  for (int i = 0; i < kRopeMaxPairs; ++i) {
    t->turn[i] = 0;
    t->axis[i] = 0;
  }
  for (int i = 0; i < rot / 2; ++i) {
    const double f = rope->inv_freq[i];
    if (!(std::fabs(f) < 2147483648.0))
      return fail(MA_ERR_INVALID_ARG, "inv_freq[%d] = %g", i, f);
    t->turn[i] = turn_per_position(f);
    const int32_t a = rope->axis ? rope->axis[i] : 0;
    if (a < 0 || a >= rope->num_axes)
      return fail(MA_ERR_INVALID_ARG, "axis[%d] = %d outside [0, %d)", i, a,
                  rope->num_axes);
    t->axis[i] = static_cast<uint8_t>(a);
  }
  return MA_OK;
}

}  // namespace host
}  // namespace mesh_attn
