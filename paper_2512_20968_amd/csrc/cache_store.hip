// Rows of K and V into the 4-bit cache and back (mesh_attn_cache_append,
// mesh_attn_cache_read).
//
// A group of 32 dims shares the scale 2^e, the least power of two with amax <=
// 7 * 2^e: an element in (6, 7] of those units rounds to 6, within half a step,
// while a scale one smaller would cut up to a quarter off the largest element.
// Scaling by a power of two is exact in float32, so the hardware's conversion
// to E2M1 (nearest, ties to even, saturating) makes the only rounding.
//
// Both directions are streaming kernels: 4 d bytes of bf16 and d + d/16 bytes
// of cache per (token, KV head).  A thread holds 8 dims of one (row, head) of K
// and of V: 16 bytes of bf16 each, 4 bytes of codes each; four neighbouring
// lanes hold a group.  32768 rows of 8 heads of 128: append 37 us, 4.6 TB/s,
// read 27 us, 6.3 TB/s, where a large copy has 5.35; 64 rows 3 us each, of which
// nearly all is the launch.  Four rows per thread, their loads in flight
// together, are slower at every size (append 38.4, read 27.2 us; 4096 rows 7.0 and
// 5.3 us instead of 6.0 and 4.5): waves enough are there all the same.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_codes.h"

namespace mesh_attn {
namespace {

using namespace dev;

constexpr int NT = 256;

__device__ __forceinline__ Quant quantize8(u32x4 raw) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(raw[i] << 16);
    x[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
  }
  return dev::quantize8(x);
}

// Threads take (row, head, chunk of 8 dims), chunks fastest, then rows: a
// workgroup's rows are one head's, next to each other in the cache where their
// slots are.
template <int D>
constexpr int kRows = NT / (D / 8);

// A launch counts its threads in 32 bits per dimension: many workgroups of rows
// go on in z.
constexpr int64_t kMaxGridX = 1 << 22;

template <int D>
__device__ __forceinline__ int64_t thread_row() {
  return (int64_t{blockIdx.z} * gridDim.x + blockIdx.x) * kRows<D> +
         threadIdx.x / (D / 8);
}

template <int D>
__global__ __launch_bounds__(NT) void cache_append_kernel(StoreParams p) {
  const int64_t row = thread_row<D>();
  if (row >= p.rows) return;  // a group's four lanes alike
  const int lg = p.c.page_log2, chunk = threadIdx.x % (D / 8);
  const int head = blockIdx.y;
  const int64_t col = int64_t{head} * D + chunk * 8;
  const int64_t slot = p.slots[row];
  const Quant k = quantize8(
      *reinterpret_cast<const u32x4*>(p.k + row * p.k_stride + col));
  const Quant v = quantize8(
      *reinterpret_cast<const u32x4*>(p.v + row * p.v_stride + col));
  if (slot < 0 || slot >= int64_t{p.c.num_pages} << lg) return;
  const int t = static_cast<int>(slot & (p.c.page_size() - 1));
  uint8_t* blk = p.data + ((slot >> lg) * p.c.hkv + head) *
                              int64_t{p.c.block_bytes()};
  store_quants<D>(blk, lg, t, chunk, k, v);
}

__device__ __forceinline__ u32x4 values8(uint32_t codes, uint32_t scale) {
  const uint32_t nan2 = 0x7fc07fc0u;
  const u32x4 nan = {nan2, nan2, nan2, nan2};
  const u32x4 x =
      __builtin_bit_cast(u32x4, dequant8(codes, scale_of(scale)));
  return scale == kScaleNaN ? nan : x;
}

template <int D>
__global__ __launch_bounds__(NT) void cache_read_kernel(LoadParams p) {
  using B = Block<D>;
  const int64_t row = thread_row<D>();
  if (row >= p.rows) return;
  const int lg = p.c.page_log2, chunk = threadIdx.x % (D / 8);
  const int head = blockIdx.y;
  const int64_t slot = p.slots[row];
  u32x4 k = {0, 0, 0, 0}, v = k;
  if (slot >= 0 && slot < int64_t{p.c.num_pages} << lg) {
    const int t = static_cast<int>(slot & (p.c.page_size() - 1));
    const uint8_t* blk = p.data + ((slot >> lg) * p.c.hkv + head) *
                                      int64_t{p.c.block_bytes()};
    const uint32_t kc =
        *reinterpret_cast<const uint32_t*>(blk + B::k_codes(lg, t) + chunk * 4);
    uint32_t vc;
    if constexpr (D == 128) {
      vc = *reinterpret_cast<const uint32_t*>(blk + B::v_codes(lg, t, chunk));
    } else {
      vc = *reinterpret_cast<const uint16_t*>(blk +
                                              B::v_codes(lg, t, 2 * chunk)) |
           uint32_t{*reinterpret_cast<const uint16_t*>(
               blk + B::v_codes(lg, t, 2 * chunk + 1))}
               << 16;
    }
    k = values8(kc, blk[B::k_scale(lg, t, chunk / 4)]);
    v = values8(vc, blk[B::v_scale(lg, t, chunk / 4)]);
  }
  const int64_t at = (row * p.c.hkv + head) * D + chunk * 8;
  __builtin_nontemporal_store(k, reinterpret_cast<u32x4*>(p.k + at));
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(p.v + at));
}

template <int D>
dim3 grid_of(int64_t rows, int hkv) {
  const int64_t groups = (rows + kRows<D> - 1) / kRows<D>;
  const int64_t x = groups < kMaxGridX ? groups : kMaxGridX;
  return dim3(static_cast<unsigned>(x), static_cast<unsigned>(hkv),
              static_cast<unsigned>((groups + x - 1) / x));
}

template <int D>
void append(const StoreParams& p, hipStream_t stream) {
  hipLaunchKernelGGL(cache_append_kernel<D>, grid_of<D>(p.rows, p.c.hkv),
                     dim3(NT), 0, stream, p);
}

template <int D>
void read(const LoadParams& p, hipStream_t stream) {
  hipLaunchKernelGGL(cache_read_kernel<D>, grid_of<D>(p.rows, p.c.hkv),
                     dim3(NT), 0, stream, p);
}

}  // namespace

hipError_t launch_cache_append(const StoreParams& p, hipStream_t stream) {
  p.c.d == 128 ? append<128>(p, stream) : append<64>(p, stream);
  return hipGetLastError();
}

hipError_t launch_cache_read(const LoadParams& p, hipStream_t stream) {
  p.c.d == 128 ? read<128>(p, stream) : read<64>(p, stream);
  return hipGetLastError();
}

}  // namespace mesh_attn
