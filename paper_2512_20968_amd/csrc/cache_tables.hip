// Block tables, slots and positions of a step, built on the device from the
// requests' lengths (mesh_attn_cache_tables).
//
// The pages a request takes follow from prefix sums over the requests (new
// rows; pages wanted), the rest is one lookup per row and per new page.  A
// launch is bound by latency, not by its few hundred KB: so every workgroup
// makes the prefix sums for itself in LDS (they are at most 4096 requests, 16 a
// thread) and takes a share of the rows and new pages, and there is one launch
// and no workspace.  No workgroup reads what another writes: block table
// entries below a request's old pages are only read, those from there on only
// written (a row on a new page takes its number from the free list).

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache.h"

namespace mesh_attn {
namespace {

constexpr int NT = 256;
constexpr int kWaves = NT / 64;
constexpr uint32_t kTop = 0x7fffffffu;  // sums are capped here
constexpr int32_t kRefused = INT32_MIN;

// Capped addition of numbers up to kTop: associative, so a scan may use it.
__device__ __forceinline__ uint32_t add_capped(uint32_t a, uint32_t b) {
  return min(a + b, kTop);
}

struct Request {
  int32_t len, add;       // tokens so far and new ones
  int32_t before, after;  // pages of its stored tokens, without and with them
  bool fits;
};

__device__ __forceinline__ Request load_request(const TablesParams& p, int b) {
  Request r;
  r.len = max(p.lens[b], 0);
  r.add = max(p.new_lens[b], 0);
  const int ps = p.c.page_size();
  const int64_t total = int64_t{r.len} + r.add;
  r.before = (p.c.share.below(r.len) + int64_t{ps} - 1) >> p.c.page_log2;
  r.fits = total <= int64_t{kTop};
  r.after = r.fits ? static_cast<int32_t>(
                         (p.c.share.below(total) + int64_t{ps} - 1) >>
                         p.c.page_log2)
                   : r.before;
  r.fits = r.fits && r.after <= p.c.max_pages;
  return r;
}

// Last index i of a[0 .. n) with a[i] <= x, a increasing and a[0] <= x.
__device__ __forceinline__ int last_not_above(const int32_t* a, int n,
                                              int64_t x) {
  int lo = 0, hi = n;  // a[lo] <= x < a[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if ((a[mid] & kTop) <= x)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// Exclusive capped prefix sum of `x` over the workgroup's threads; *total is
// the sum over all.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* s_wave,
                                               uint32_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t y = x;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const uint32_t z = __shfl_up(y, o);
    if (lane >= o) y = add_capped(y, z);
  }
  uint32_t before = __shfl_up(y, 1);
  if (lane == 0) before = 0;
  if (lane == 63) s_wave[wave] = y;
  __syncthreads();
  uint32_t base = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) base = sum;
    sum = add_capped(sum, s_wave[w]);
  }
  __syncthreads();
  *total = sum;
  return add_capped(base, before);
}

__global__ __launch_bounds__(NT) void cache_tables_kernel(TablesParams p) {
  extern __shared__ int32_t lds[];
  const int B = p.num_requests, tid = threadIdx.x;
  int32_t* s_cu = lds;             // [B + 1] first row
  int32_t* s_page = lds + B + 1;   // [B + 1] first new page; bit 31: refused
  __shared__ uint32_t s_wave[kWaves];
  __shared__ int s_refused;
  if (tid == 0) s_refused = 0;

  const int per = (B + NT - 1) / NT;
  const int b0 = min(tid * per, B), b1 = min(b0 + per, B);
  const int first = min(max(p.free_range[0], 0), p.num_free);
  const int last = min(max(p.free_range[1], first), p.num_free);
  uint32_t rows = 0, want = 0;
  for (int b = b0; b < b1; ++b) {
    const Request r = load_request(p, b);
    rows = add_capped(rows, r.add);
    if (r.fits) want = add_capped(want, r.after - r.before);
  }
  uint32_t rows_total, want_total;
  rows = block_scan(rows, s_wave, &rows_total);
  want = block_scan(want, s_wave, &want_total);

  // Requests: where their rows and pages start, and whether they get them.
  const uint32_t avail = last - first;
  int taken = 0, refused = 0;
  for (int b = b0; b < b1; ++b) {
    const Request r = load_request(p, b);
    const uint32_t mine = r.fits ? r.after - r.before : 0;
    const uint32_t end = add_capped(want, mine);
    const bool ok = r.fits && (mine == 0 || end <= avail);
    s_cu[b] = rows;
    s_page[b] = static_cast<int32_t>(want) | (ok ? 0 : kRefused);
    if (ok && mine > 0) taken = end;
    if (!ok) ++refused;
    if (blockIdx.x == 0) {
      p.cu_new[b] = rows;
      p.lens_out[b] = ok ? r.len + r.add : p.lens[b];
    }
    rows = add_capped(rows, r.add);
    want = end;
  }
  if (tid == 0) {
    s_cu[B] = rows_total;
    s_page[B] = want_total;
  }
  if (refused) atomicAdd(&s_refused, refused);
  // The accepted requests' pages are a prefix of those wanted: the largest end
  // is their number.
#pragma unroll
  for (int o = 32; o > 0; o /= 2) taken = max(taken, __shfl_xor(taken, o));
  __syncthreads();
  if ((tid & 63) == 0) s_wave[tid >> 6] = taken;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) taken = max(taken, int(s_wave[w]));
  if (blockIdx.x == 0 && tid == 0) {
    p.cu_new[B] = rows_total;
    p.free_range_out[0] = first + taken;
    p.free_range_out[1] = last;
    *p.refused = s_refused;
  }

  const int64_t at0 = int64_t{blockIdx.x} * NT + tid;
  const int64_t step = int64_t{gridDim.x} * NT;
  // New pages.
  for (int64_t j = at0; j < taken; j += step) {
    const int b = last_not_above(s_page, B, j);
    if (s_page[b] < 0) continue;
    const int32_t before =
        (p.c.share.below(max(p.lens[b], 0)) + int64_t{p.c.page_size()} - 1) >>
        p.c.page_log2;
    p.block_table[int64_t{b} * p.c.max_pages + before + (j - s_page[b])] =
        p.free_pages[first + j];
  }
  // Rows.
  for (int64_t r = at0; r < p.rows; r += step) {
    int64_t slot = -1;
    int32_t pos = -1;
    if (r < rows_total) {
      const int b = last_not_above(s_cu, B, r);
      const int32_t page_first = s_page[b];
      if (page_first >= 0) {
        const int32_t len = max(p.lens[b], 0);
        pos = len + static_cast<int32_t>(r - s_cu[b]);
        const int32_t local = p.c.share.below(pos);
        if (p.c.share.below(int64_t{pos} + 1) > local) {
          const int32_t before =
              (p.c.share.below(len) + int64_t{p.c.page_size()} - 1) >>
              p.c.page_log2;
          const int32_t i = local >> p.c.page_log2;
          const int32_t page =
              i < before ? p.block_table[int64_t{b} * p.c.max_pages + i]
                         : p.free_pages[first + page_first + (i - before)];
          if (page >= 0 && page < p.c.num_pages)
            slot = (int64_t{page} << p.c.page_log2) +
                   (local & (p.c.page_size() - 1));
        }
      }
    }
    p.slots[r] = slot;
    p.positions[r] = pos;
  }
}

}  // namespace

hipError_t launch_cache_tables(const TablesParams& p, hipStream_t stream) {
  // Four rows a thread: one workgroup makes a decode step's tables.
  int64_t grid = (p.rows + 4 * NT - 1) / (4 * NT);
  if (grid < 1) grid = 1;
  if (grid > 512) grid = 512;
  const size_t lds = (2 * static_cast<size_t>(p.num_requests) + 2) * 4;
  hipLaunchKernelGGL(cache_tables_kernel, dim3(static_cast<unsigned>(grid)),
                     dim3(NT), lds, stream, p);
  return hipGetLastError();
}

}  // namespace mesh_attn
