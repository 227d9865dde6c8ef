// Rotary positions with several axes (mesh_attn_rope).
//
// A pair turns by position * frequency.  The host gives every pair's turn per
// position as a 64-bit fraction of a full turn; multiplied by the position
// modulo 2^64 this is the angle's exact fraction of a turn to 2^31 * 2^-64,
// where a float32 angle of a position near a million has lost five digits.  The
// fraction's top two bits after rounding are the quadrant, the rest (at most an
// eighth of a turn) goes to sincospi in float32.
//
// Streaming: every element is read and written once.  A thread owns one 16-byte
// unit's worth of pairs of a row, makes their angles once and walks over heads of
// Q and K, four at a time with all their loads in flight.

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

// cos and sin of a turn by per * pos (2^-64 turns, modulo 1).
__device__ __forceinline__ void turn_of(uint64_t per, int32_t pos, float* c,
                                        float* s) {
  const uint64_t frac = per * static_cast<uint64_t>(int64_t{pos});
  // Quadrant, and the signed rest in 2^-64 turns: at most an eighth.
  const uint64_t near = frac + (uint64_t{1} << 61);
  const uint32_t quad = static_cast<uint32_t>(near >> 62);
  const int64_t rest =
      static_cast<int64_t>(frac - (static_cast<uint64_t>(quad) << 62));
  // Radians, |t| <= pi / 4: 2 pi 2^-34 a unit of the rest's upper bits.
  const float t = static_cast<float>(static_cast<int32_t>(rest >> 30)) *
                  static_cast<float>(6.283185307179586 * 0x1p-34);
  // Taylor: the first terms left out are below 2^-29 of sin and 2^-33 of cos.
  const float z = t * t;
  float sn = fmaf(z, 1.f / 362880, -1.f / 5040);
  sn = fmaf(sn, z, 1.f / 120);
  sn = fmaf(sn, z, -1.f / 6);
  sn = fmaf(sn * z, t, t);
  float cs = fmaf(z, -1.f / 3628800, 1.f / 40320);
  cs = fmaf(cs, z, -1.f / 720);
  cs = fmaf(cs, z, 1.f / 24);
  cs = fmaf(cs, z, -0.5f);
  cs = fmaf(cs, z, 1.f);
  const float a = (quad & 1) ? sn : cs, b = (quad & 1) ? cs : sn;
  *c = (quad == 1 || quad == 2) ? -a : a;
  *s = (quad & 2) ? -b : b;
}

// Heads loaded together.
constexpr int kBatch = 4;

// The units of a head are rotated ones (two per thread and head: units i and
// i + rot/2 of the halves, or, interleaved, two neighbours), then copied ones.
// blockIdx.y: p.batches * kBatch heads of Q's, then K's.
template <bool F32, bool INTER>
__global__ __launch_bounds__(NT) void rope_kernel(RopeParams p) {
  constexpr int N = Unit<F32>::N;
  const int half = p.rot / 2;
  const uint32_t rot_units = half / N,
                 units = rot_units + (p.d - p.rot) / N;
  const int64_t total = p.rows * units;
  const int64_t idx = int64_t{blockIdx.x} * NT + threadIdx.x;
  if (idx >= total) return;
  const int64_t row = total < (int64_t{1} << 32)
                          ? int64_t{uint32_t(idx) / units}
                          : idx / units;
  const uint32_t u = static_cast<uint32_t>(idx - row * units);
  const bool turns = u < rot_units;
  float c[N], s[N];
  int at0, at1;
  if (turns) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int pair = u * N + j;
      turn_of(p.t.turn[pair], p.positions[p.t.axis[pair] * p.rows + row], &c[j],
              &s[j]);
      if (p.inverse) s[j] = -s[j];
    }
    at0 = INTER ? 2 * u * N : u * N;
    at1 = INTER ? at0 + N : at0 + half;
  } else {
    at0 = at1 = p.rot + (u - rot_units) * N;
  }
  const int heads = p.heads[0] + p.heads[1];
  int h0 = blockIdx.y * (p.batches * kBatch);
  for (int b = 0; b < p.batches && h0 < heads; ++b, h0 += kBatch) {
    float x[kBatch][2 * N];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int h = min(h0 + i, heads - 1), t = h < p.heads[0] ? 0 : 1;
      const int64_t in = row * p.x_stride[t] +
                         int64_t{t ? h - p.heads[0] : h} * p.d;
      Unit<F32>::load(p.x[t], in + at0, x[i]);
      if (turns) Unit<F32>::load(p.x[t], in + at1, x[i] + N);
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int h = h0 + i, t = h < p.heads[0] ? 0 : 1;
      if (h >= heads) break;
      const int64_t out = row * p.y_stride[t] +
                          int64_t{t ? h - p.heads[0] : h} * p.d;
      if (turns) {
        float y[2 * N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const int a = INTER ? 2 * j : j, e = INTER ? 2 * j + 1 : j + N;
          y[a] = x[i][a] * c[j] - x[i][e] * s[j];
          y[e] = x[i][e] * c[j] + x[i][a] * s[j];
        }
        Unit<F32>::store(p.y[t], out + at0, y);
        Unit<F32>::store(p.y[t], out + at1, y + N);
      } else if (p.x[t] != p.y[t]) {
        Unit<F32>::store(p.y[t], out + at0, x[i]);
      }
    }
  }
}

}  // namespace

hipError_t launch_rope(const RopeParams& params, bool f32,
                       hipStream_t stream) {
  RopeParams p = params;
  const int n = f32 ? 4 : 8;
  const int units = p.rot / 2 / n + (p.d - p.rot) / n;
  const int64_t grid = (p.rows * units + NT - 1) / NT;
  // Angles are made once for all the heads of a thread, of which more threads
  // have fewer.
  const int batches = (p.heads[0] + p.heads[1] + kBatch - 1) / kBatch;
  p.batches = 1;
  while (p.batches < 4 && grid * (batches / (2 * p.batches)) >= 2048)
    p.batches *= 2;
  const dim3 g(static_cast<unsigned>(grid),
               (batches + p.batches - 1) / p.batches);
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
