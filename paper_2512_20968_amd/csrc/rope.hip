// Rotary positions with several axes (mesh_attn_rope).
//
// A pair turns by position * frequency.  The host gives every pair's turn per
// position as a 64-bit fraction of a full turn; multiplied by the position
// modulo 2^64 this is the angle's exact fraction of a turn to 2^31 * 2^-64,
// where a float32 angle of a position near a million has lost five digits.  The
// fraction's top two bits after rounding are the quadrant, the rest (at most an
// eighth of a turn) goes to sincospi in float32.
//
// Streaming: every element is read and written once, the angles are made once
// per (row, pair) and used for all heads of Q and K.  A thread owns one
// 16-byte unit's worth of pairs of a row and walks over the heads.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache.h"

namespace mesh_attn {
namespace {

constexpr int NT = 256;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes of a head as float32.
template <bool F32>
struct Unit;
template <>
struct Unit<true> {
  static constexpr int N = 4;
  static __device__ void load(const void* base, int64_t i, float* x) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(
        static_cast<const float*>(base) + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = v[j];
  }
  static __device__ void store(void* base, int64_t i, const float* x) {
    f32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = x[j];
    *reinterpret_cast<f32x4*>(static_cast<float*>(base) + i) = v;
  }
};
template <>
struct Unit<false> {
  static constexpr int N = 8;
  typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
  static __device__ void load(const void* base, int64_t i, float* x) {
    const bf16x8 v = *reinterpret_cast<const bf16x8*>(
        static_cast<const __bf16*>(base) + i);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = static_cast<float>(v[j]);
  }
  static __device__ void store(void* base, int64_t i, const float* x) {
    bf16x8 v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = static_cast<__bf16>(x[j]);
    *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(base) + i) = v;
  }
};

__device__ __forceinline__ void turn_of(uint64_t per, int32_t pos, float* c,
                                        float* s) {
  const uint64_t frac = per * static_cast<uint64_t>(int64_t{pos});
  // Quadrant, and the signed rest in 2^-64 turns.
  const uint64_t near = frac + (uint64_t{1} << 61);
  const uint32_t quad = static_cast<uint32_t>(near >> 62);
  const int64_t rest =
      static_cast<int64_t>(frac - (static_cast<uint64_t>(quad) << 62));
  // Half turns: rest * 2^-63, |.| <= 1/4.
  const float x = static_cast<float>(static_cast<int32_t>(rest >> 30)) *
                  0x1p-33f;
  float sn, cs;
  sincospif(x, &sn, &cs);
  const float a = (quad & 1) ? sn : cs, b = (quad & 1) ? cs : sn;
  *c = (quad == 1 || quad == 2) ? -a : a;
  *s = (quad & 2) ? -b : b;
}

// The units of a head are rotated ones (two per thread and step: the halves'
// units i and i + rot/2, or, interleaved, two neighbours), then copied ones.
template <bool F32, bool INTER>
__global__ __launch_bounds__(NT) void rope_kernel(RopeParams p) {
  constexpr int N = Unit<F32>::N;
  const int half = p.rot / 2;
  const int rot_units = half / N, units = rot_units + (p.d - p.rot) / N;
  const int64_t total = p.rows * units;
  const int64_t idx = int64_t{blockIdx.x} * NT + threadIdx.x;
  if (idx >= total) return;
  const int64_t row = idx / units;
  const int u = static_cast<int>(idx - row * units);
  if (u >= rot_units) {
    const int at = p.rot + (u - rot_units) * N;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (p.x[t] == p.y[t]) continue;
      for (int h = 0; h < p.heads[t]; ++h) {
        float x[N];
        Unit<F32>::load(p.x[t], row * p.x_stride[t] + h * p.d + at, x);
        Unit<F32>::store(p.y[t], row * p.y_stride[t] + h * p.d + at, x);
      }
    }
    return;
  }
  float c[N], s[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int pair = u * N + j;
    turn_of(p.t.turn[pair], p.positions[p.t.axis[pair] * p.rows + row], &c[j],
            &s[j]);
    if (p.inverse) s[j] = -s[j];
  }
  const int at0 = INTER ? 2 * u * N : u * N;
  const int at1 = INTER ? at0 + N : at0 + half;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    for (int h = 0; h < p.heads[t]; ++h) {
      float x[2 * N], y[2 * N];
      const int64_t in = row * p.x_stride[t] + h * p.d;
      const int64_t out = row * p.y_stride[t] + h * p.d;
      Unit<F32>::load(p.x[t], in + at0, x);
      Unit<F32>::load(p.x[t], in + at1, x + N);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int a = INTER ? 2 * j : j, b = INTER ? 2 * j + 1 : j + N;
        y[a] = x[a] * c[j] - x[b] * s[j];
        y[b] = x[b] * c[j] + x[a] * s[j];
      }
      Unit<F32>::store(p.y[t], out + at0, y);
      Unit<F32>::store(p.y[t], out + at1, y + N);
    }
  }
}

}  // namespace

hipError_t launch_rope(const RopeParams& p, bool f32, hipStream_t stream) {
  const int n = f32 ? 4 : 8;
  const int units = p.rot / 2 / n + (p.d - p.rot) / n;
  const int64_t grid = (p.rows * units + NT - 1) / NT;
  const dim3 g(static_cast<unsigned>(grid));
  if (f32) {
    if (p.interleaved)
      hipLaunchKernelGGL((rope_kernel<true, true>), g, dim3(NT), 0, stream, p);
    else
      hipLaunchKernelGGL((rope_kernel<true, false>), g, dim3(NT), 0, stream, p);
  } else {
    if (p.interleaved)
      hipLaunchKernelGGL((rope_kernel<false, true>), g, dim3(NT), 0, stream, p);
    else
      hipLaunchKernelGGL((rope_kernel<false, false>), g, dim3(NT), 0, stream,
                         p);
  }
  return hipGetLastError();
}

}  // namespace mesh_attn
