// Internal interface of the 4-bit key/value cache and of rotary positions:
// what the host (cache.cpp) passes to the kernels.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mesh_attn {

// Caps above this are wide ones: a capped score made as cap - 2 cap r is off by
// 2^-23 of the cap (2^-15 of one up to here, 2^-7 of a bf16 weight's rounding),
// whatever its own size; under a wide cap small arguments of the tanh take its
// series.
constexpr float kWideCap = 256.f;

// Which positions of a sequence a cache stores, and how many of them lie below
// a position.
struct CacheShare {
  int32_t striped, n, p;
  int64_t first, len;  // contiguous: [first, first + len)

  // Number of stored positions < x, for x up to 2^31; at most 2^31 - 1.
  __host__ __device__ int32_t below(int64_t x) const {
    if (striped) {
      if (x <= p) return 0;
      if (n == 1) return static_cast<int32_t>(x < INT32_MAX ? x : INT32_MAX);
      // x - p + n - 1 < 2^31 + 2^31.
      return static_cast<int32_t>(static_cast<uint32_t>(x - p + n - 1) /
                                  static_cast<uint32_t>(n));
    }
    const int64_t y = x - first;
    return static_cast<int32_t>(y < 0 ? 0 : y > len ? len : y);
  }
};

struct CacheDims {
  CacheShare share;
  int32_t num_pages, page_log2, hkv, d, max_pages;

  __host__ __device__ int32_t page_size() const { return 1 << page_log2; }
  // Bytes of a (page, KV head) block.
  __host__ __device__ int32_t block_bytes() const {
    return (d + d / 16) << page_log2;
  }
};

struct TablesParams {
  CacheDims c;
  const int32_t* lens;
  const int32_t* new_lens;
  const int32_t* free_pages;
  const int32_t* free_range;
  int32_t* block_table;
  int32_t* lens_out;
  int32_t* cu_new;
  int64_t* slots;
  int32_t* positions;
  int32_t* free_range_out;
  int32_t* refused;
  int64_t rows;
  int32_t num_requests, num_free;
};
hipError_t launch_cache_tables(const TablesParams& p, hipStream_t stream);

struct StoreParams {
  CacheDims c;
  const uint16_t* k;
  const uint16_t* v;
  int64_t k_stride, v_stride;
  const int64_t* slots;
  uint8_t* data;
  int64_t rows;
};
hipError_t launch_cache_append(const StoreParams& p, hipStream_t stream);

struct LoadParams {
  CacheDims c;
  const int64_t* slots;
  const uint8_t* data;
  uint16_t* k;
  uint16_t* v;
  int64_t rows;
};
hipError_t launch_cache_read(const LoadParams& p, hipStream_t stream);

// A sequence of the attention whose partial results are to be joined: those of
// `parts` runs from `start` on (0: none).
struct CacheFold {
  int32_t first, rr0, rr_end, kvh, parts, start;
};
// Its request's stored keys, under a score rule.
struct CacheFoldKeys {
  int32_t from, local;
};

struct CacheFwdParams {
  CacheDims c;
  const uint16_t* q;
  int64_t q_stride;
  const int32_t* positions;
  const int32_t* cu;
  const int32_t* lens;
  const int32_t* block_table;
  const uint8_t* data;
  void* o;
  float* lse;
  int64_t rows;
  int32_t hq, group, num_requests;
  uint32_t group_mul;   // token_head()
  int32_t group_shift;
  float scale_log2, inv_scale_log2;
  int32_t least_keys, most_keys;  // stored keys of the launch's requests
  int32_t split;      // whether sequences are cut, ..
  int32_t may_stay_whole;  // .. unless their lengths speak against it
  int32_t unit_log2;  // keys of a unit
  int32_t seq_units;  // units that a sequence costs beside its keys
  int32_t max_units;  // most of a launch
  // The score rule (rule = 1): cap_two = 2 cap log2(e), 0 without a cap; a
  // product times cap_in is log2(e^(2u)), times cap_u u = score / cap; wide_cap: the
  // kernels that take small arguments from the tanh's series.
  int32_t rule, wide_cap;
  float cap_in, cap_two, cap_u;
  const float* slopes;
  const int32_t* key_begin;
  const int32_t* key_end;
  CacheFold* fold;           // [workgroup][2]: goes on in its run, starts in it
  CacheFoldKeys* fold_keys;  // [workgroup][2]
  float* part_o;             // [2 * workgroups][rows of a tile][d]
  float* part_ml;            // .. [2]: reference (log2 units) and sum
};

hipError_t launch_cache_fwd(const CacheFwdParams& p, bool out_f32, void* ws,
                            hipStream_t stream);
size_t cache_fwd_workspace(const CacheDims& c, int32_t num_requests,
                           int64_t rows);

// One pair's turn per position, as a 64-bit fraction of a full turn, and its
// axis.
constexpr int kRopeMaxPairs = 128;
struct RopeTable {
  uint64_t turn[kRopeMaxPairs];
  uint8_t axis[kRopeMaxPairs];
};
struct RopeParams {
  RopeTable t;
  const int32_t* positions;
  const void* x[2];
  void* y[2];
  int64_t x_stride[2], y_stride[2];
  int64_t rows;
  int32_t heads[2];
  int32_t d, rot, interleaved, inverse;
  int32_t group_rows;  // rows of a workgroup
};
static_assert(sizeof(RopeParams) <= 4096, "kernel arguments");
hipError_t launch_rope(const RopeParams& p, bool f32, hipStream_t stream);

}  // namespace mesh_attn
