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
// lanes hold a group.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_codes.h"

namespace mesh_attn {
namespace {

using namespace dev;

constexpr int NT = 256;

// Codes of 8 values and their group's scale code.
struct Quant {
  uint32_t codes, scale;
};

__device__ __forceinline__ Quant quantize8(u32x4 raw) {
  float x[8];
  uint32_t top = 0;  // largest magnitude, as float bits (NaN above infinity)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = raw[i] << 16, hi = raw[i] & 0xffff0000u;
    x[2 * i] = __uint_as_float(lo);
    x[2 * i + 1] = __uint_as_float(hi);
    top = max(top, max(lo & 0x7fffffffu, hi & 0x7fffffffu));
  }
  top = max(top, uint32_t(__shfl_xor(int(top), 1)));
  top = max(top, uint32_t(__shfl_xor(int(top), 2)));
  const bool finite = top < 0x7f800000u;
  int e = int(top >> 23) - 129 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  e = min(max(e, -126), 125);
  // 2^-e; a group that is not finite gets codes of 0 and the NaN scale.
  const float inv = finite ? __uint_as_float(uint32_t(127 - e) << 23) : 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = finite ? x[i] * inv : 0.f;
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], 1.f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], 1.f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], 1.f, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], 1.f, 3);
  return {w, finite ? uint32_t(e + 127) : kScaleNaN};
}

// Threads take (row, head, chunk of 8 dims), chunks fastest, then rows, kU rows
// each with all their loads in flight: a workgroup's rows are one head's, next
// to each other in the cache where their slots are.
template <int D, int U>
__global__ __launch_bounds__(NT) void cache_append_kernel(StoreParams p) {
  constexpr int kChunks = D / 8, kRows = NT / kChunks;
  using B = Block<D>;
  const int lg = p.c.page_log2, chunk = threadIdx.x % kChunks;
  const int head = blockIdx.y;
  const int64_t slots_end = int64_t{p.c.num_pages} << lg;
  const int64_t row0 =
      int64_t{blockIdx.x} * (kRows * U) + threadIdx.x / kChunks;
  const int64_t col = int64_t{head} * D + chunk * 8;
  int64_t slot[U];
  u32x4 kr[U], vr[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int64_t row = min(row0 + i * kRows, p.rows - 1);
    slot[i] = row0 + i * kRows < p.rows ? p.slots[row] : -1;
    kr[i] = *reinterpret_cast<const u32x4*>(p.k + row * p.k_stride + col);
    vr[i] = *reinterpret_cast<const u32x4*>(p.v + row * p.v_stride + col);
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const Quant k = quantize8(kr[i]), v = quantize8(vr[i]);
    if (slot[i] < 0 || slot[i] >= slots_end) continue;
    const int t = static_cast<int>(slot[i] & (p.c.page_size() - 1));
    uint8_t* blk = p.data + ((slot[i] >> lg) * p.c.hkv + head) *
                                int64_t{p.c.block_bytes()};
    *reinterpret_cast<uint32_t*>(blk + B::k_codes(lg, t) + chunk * 4) = k.codes;
    if constexpr (D == 128) {
      *reinterpret_cast<uint32_t*>(blk + B::v_codes(lg, t, chunk)) = v.codes;
    } else {
      *reinterpret_cast<uint16_t*>(blk + B::v_codes(lg, t, 2 * chunk)) =
          static_cast<uint16_t>(v.codes);
      *reinterpret_cast<uint16_t*>(blk + B::v_codes(lg, t, 2 * chunk + 1)) =
          static_cast<uint16_t>(v.codes >> 16);
    }
    if ((chunk & 3) == 0) {
      blk[B::k_scale(lg, t, chunk / 4)] = static_cast<uint8_t>(k.scale);
      blk[B::v_scale(lg, t, chunk / 4)] = static_cast<uint8_t>(v.scale);
    }
  }
}

__device__ __forceinline__ u32x4 values8(uint32_t codes, uint32_t scale) {
  const uint32_t nan2 = 0x7fc07fc0u;
  const u32x4 nan = {nan2, nan2, nan2, nan2};
  const u32x4 x =
      __builtin_bit_cast(u32x4, dequant8(codes, scale_of(scale)));
  return scale == kScaleNaN ? nan : x;
}

template <int D, int U>
__global__ __launch_bounds__(NT) void cache_read_kernel(LoadParams p) {
  constexpr int kChunks = D / 8, kRows = NT / kChunks;
  using B = Block<D>;
  const int lg = p.c.page_log2, chunk = threadIdx.x % kChunks;
  const int head = blockIdx.y;
  const int64_t slots_end = int64_t{p.c.num_pages} << lg;
  const int64_t row0 =
      int64_t{blockIdx.x} * (kRows * U) + threadIdx.x / kChunks;
  bool ok[U];
  uint32_t kc[U], vc[U], ks[U], vs[U];
  int64_t slot[U];
#pragma unroll
  for (int i = 0; i < U; ++i)
    slot[i] = p.slots[min(row0 + i * kRows, p.rows - 1)];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    ok[i] = slot[i] >= 0 && slot[i] < slots_end;
    const int64_t at = ok[i] ? slot[i] : 0;  // some slot's bytes
    const int t = static_cast<int>(at & (p.c.page_size() - 1));
    const uint8_t* blk =
        p.data + ((at >> lg) * p.c.hkv + head) * int64_t{p.c.block_bytes()};
    kc[i] =
        *reinterpret_cast<const uint32_t*>(blk + B::k_codes(lg, t) + chunk * 4);
    if constexpr (D == 128) {
      vc[i] = *reinterpret_cast<const uint32_t*>(blk + B::v_codes(lg, t, chunk));
    } else {
      vc[i] = *reinterpret_cast<const uint16_t*>(blk +
                                                 B::v_codes(lg, t, 2 * chunk)) |
              uint32_t{*reinterpret_cast<const uint16_t*>(
                  blk + B::v_codes(lg, t, 2 * chunk + 1))}
                  << 16;
    }
    ks[i] = blk[B::k_scale(lg, t, chunk / 4)];
    vs[i] = blk[B::v_scale(lg, t, chunk / 4)];
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    if (row0 + i * kRows >= p.rows) break;
    const u32x4 zero = {0, 0, 0, 0};
    const int64_t at = ((row0 + i * kRows) * p.c.hkv + head) * D + chunk * 8;
    __builtin_nontemporal_store(ok[i] ? values8(kc[i], ks[i]) : zero,
                                reinterpret_cast<u32x4*>(p.k + at));
    __builtin_nontemporal_store(ok[i] ? values8(vc[i], vs[i]) : zero,
                                reinterpret_cast<u32x4*>(p.v + at));
  }
}

// Rows of a workgroup's step, and whether a thread takes four of them: not
// before every compute unit has several workgroups all the same.
template <int D>
constexpr int kStepRows = NT / (D / 8);

template <int D>
bool four_rows(int64_t rows, int hkv) {
  return rows * hkv >= int64_t{4} * kStepRows<D> * 2048;
}

template <int D, int U>
dim3 grid_of(int64_t rows, int hkv) {
  constexpr int kRows = kStepRows<D> * U;
  return dim3(static_cast<unsigned>((rows + kRows - 1) / kRows), hkv);
}

template <int D>
void append(const StoreParams& p, hipStream_t stream) {
  if (four_rows<D>(p.rows, p.c.hkv))
    hipLaunchKernelGGL((cache_append_kernel<D, 4>),
                       (grid_of<D, 4>(p.rows, p.c.hkv)), dim3(NT), 0, stream, p);
  else
    hipLaunchKernelGGL((cache_append_kernel<D, 1>),
                       (grid_of<D, 1>(p.rows, p.c.hkv)), dim3(NT), 0, stream, p);
}

template <int D>
void read(const LoadParams& p, hipStream_t stream) {
  if (four_rows<D>(p.rows, p.c.hkv))
    hipLaunchKernelGGL((cache_read_kernel<D, 4>),
                       (grid_of<D, 4>(p.rows, p.c.hkv)), dim3(NT), 0, stream, p);
  else
    hipLaunchKernelGGL((cache_read_kernel<D, 1>),
                       (grid_of<D, 1>(p.rows, p.c.hkv)), dim3(NT), 0, stream, p);
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
