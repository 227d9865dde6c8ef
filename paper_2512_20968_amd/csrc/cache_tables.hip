// Block tables, slots and positions of a step, built on the device from the
// requests' lengths (mesh_attn_cache_tables).
//
// The pages a request takes follow from prefix sums over the requests (new
// rows; pages wanted), the rest is one lookup per row and per new page.  A
// launch is bound by latency, not by its few hundred KB: so every workgroup
// makes the prefix sums for itself in LDS (they are at most 4096 requests, 16 a
// thread) and takes a share of the rows and new pages, and there is one launch
// and no workspace: 3.2 us for 40 requests of one new token, of which 2.5 are the
// launch, 7.0 us for 700 requests with 17 thousand new tokens.  No workgroup
// reads what another writes: block table entries below a request's old pages are
// only read, those from there on only written (a row on a new page takes its
// number from the free list).

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

// What the rows and pages of a request need, in LDS.
struct Kept {
  int32_t row, page;   // first row; first new page, bit 31: refused
  int32_t len, before;
};

// Last request i of n whose `field` (without bit 31) is at most x; the field
// does not decrease, and the first one's is at most x.
__device__ __forceinline__ int last_not_above(const Kept* a,
                                              int32_t Kept::*field, int n,
                                              int64_t x) {
  int lo = 0, hi = n;  // lo's is at most x, hi's above
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if ((a[mid].*field & int32_t(kTop)) <= x)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// Exclusive capped prefix sums of x[0] and x[1] over the workgroup's threads, in
// place; total[] are the sums over all.
__device__ __forceinline__ void block_scan(uint32_t (&x)[2],
                                           uint32_t (*s_wave)[2],
                                           uint32_t (&total)[2]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t y[2] = {x[0], x[1]};
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const uint32_t z0 = __shfl_up(y[0], o), z1 = __shfl_up(y[1], o);
    if (lane >= o) {
      y[0] = add_capped(y[0], z0);
      y[1] = add_capped(y[1], z1);
    }
  }
  x[0] = __shfl_up(y[0], 1);
  x[1] = __shfl_up(y[1], 1);
  if (lane == 0) x[0] = x[1] = 0;
  if (lane == 63) {
    s_wave[wave][0] = y[0];
    s_wave[wave][1] = y[1];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    uint32_t base = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w == wave) base = sum;
      sum = add_capped(sum, s_wave[w][k]);
    }
    x[k] = add_capped(base, x[k]);
    total[k] = sum;
  }
}

__global__ __launch_bounds__(NT) void cache_tables_kernel(TablesParams p) {
  extern __shared__ Kept s_req[];  // [B + 1]
  const int B = p.num_requests, tid = threadIdx.x;
  __shared__ uint32_t s_wave[kWaves][2];
  __shared__ int s_refused, s_taken;
  if (tid == 0) s_refused = s_taken = 0;

  // Request b is thread b / per's: up to kHeld of them stay in registers.
  constexpr int kHeld = 4;
  const int per = (B + NT - 1) / NT;
  const int b0 = min(tid * per, B), b1 = min(b0 + per, B);
  const int first = min(max(p.free_range[0], 0), p.num_free);
  const int last = min(max(p.free_range[1], first), p.num_free);
  Request held[kHeld];
  uint32_t sum[2] = {0, 0}, total[2];  // rows, wanted pages
  auto count = [&](const Request& r) {
    sum[0] = add_capped(sum[0], r.add);
    if (r.fits) sum[1] = add_capped(sum[1], r.after - r.before);
  };
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (b0 + i < b1) held[i] = load_request(p, b0 + i);
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (b0 + i < b1) count(held[i]);
  for (int b = b0 + kHeld; b < b1; ++b) count(load_request(p, b));
  block_scan(sum, s_wave, total);
  uint32_t rows = sum[0], want = sum[1];

  // Requests: where their rows and pages start, and whether they get them.
  const uint32_t avail = last - first;
  int taken = 0, refused = 0;
  auto place = [&](const Request& r, int b) {
    const uint32_t mine = r.fits ? r.after - r.before : 0;
    const uint32_t end = add_capped(want, mine);
    const bool ok = r.fits && (mine == 0 || end <= avail);
    s_req[b] = Kept{static_cast<int32_t>(rows),
                    static_cast<int32_t>(want) | (ok ? 0 : kRefused), r.len,
                    r.before};
    if (ok && mine > 0) taken = end;
    if (!ok) ++refused;
    if (blockIdx.x == 0) {
      p.cu_new[b] = rows;
      p.lens_out[b] = ok ? r.len + r.add : p.lens[b];
    }
    rows = add_capped(rows, r.add);
    want = end;
  };
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (b0 + i < b1) place(held[i], b0 + i);
  for (int b = b0 + kHeld; b < b1; ++b) place(load_request(p, b), b);
  const uint32_t rows_total = total[0];
  // The accepted requests' pages are a prefix of those wanted: the largest end
  // is their number.
  if (refused) atomicAdd(&s_refused, refused);
  if (taken) atomicMax(&s_taken, taken);
  __syncthreads();
  taken = s_taken;
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
    const int b = last_not_above(s_req, &Kept::page, B, j);
    const Kept r = s_req[b];
    if (r.page < 0) continue;
    p.block_table[int64_t{b} * p.c.max_pages + r.before + (j - r.page)] =
        p.free_pages[first + j];
  }
  // Rows.
  for (int64_t i = at0; i < p.rows; i += step) {
    int64_t slot = -1;
    int32_t pos = -1;
    if (i < rows_total) {
      const int b = last_not_above(s_req, &Kept::row, B, i);
      const Kept r = s_req[b];
      if (r.page >= 0) {
        pos = r.len + static_cast<int32_t>(i - r.row);
        const int32_t local = p.c.share.below(pos);
        if (p.c.share.below(int64_t{pos} + 1) > local) {
          const int32_t n = local >> p.c.page_log2;
          const int32_t page =
              n < r.before ? p.block_table[int64_t{b} * p.c.max_pages + n]
                           : p.free_pages[first + r.page + (n - r.before)];
          if (page >= 0 && page < p.c.num_pages)
            slot = (int64_t{page} << p.c.page_log2) +
                   (local & (p.c.page_size() - 1));
        }
      }
    }
    p.slots[i] = slot;
    p.positions[i] = pos;
  }
}

}  // namespace

hipError_t launch_cache_tables(const TablesParams& p, hipStream_t stream) {
  int64_t grid = (p.rows + NT - 1) / NT;
  if (grid < 1) grid = 1;
  if (grid > 256) grid = 256;
  const size_t lds = sizeof(Kept) * (static_cast<size_t>(p.num_requests) + 1);
  hipLaunchKernelGGL(cache_tables_kernel, dim3(static_cast<unsigned>(grid)),
                     dim3(NT), lds, stream, p);
  return hipGetLastError();
}

}  // namespace mesh_attn
