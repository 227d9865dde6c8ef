// Rotary positions with several axes (mesh_attn_rope).
//
// A pair turns by position * frequency.  The host gives every pair's turn per
// position as a 64-bit fraction of a full turn, off by at most 2^-65; multiplied
// by the position modulo 2^64 this is the angle's fraction of a turn to 2^-34,
// where a float32 angle of a position near a million has lost five digits.  The
// fraction's top two bits after rounding are the quadrant; sine and cosine of the
// rest (at most an eighth of a turn) are Taylor polynomials in float32.
//
// Streaming: every element is read and written once.  A workgroup takes a few
// rows, makes each of their angles once, in LDS, and then walks over the 16-byte
// units of their heads in the order in which they lie in memory, two units
// per thread in flight.  16384 rows of 40 bf16 heads of 128 (336 MB): 63.7 us,
// 5.3 TB/s, as a large copy; with the angles made by every thread that walks
// over heads it took 72 to 79 us.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache.h"
#include "tile_common.h"

namespace mesh_attn {
namespace {

using namespace dev;

constexpr int NT = 256;

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
    __builtin_nontemporal_store(
        v, reinterpret_cast<f32x4*>(static_cast<float*>(base) + i));
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
    __builtin_nontemporal_store(
        v, reinterpret_cast<bf16x8*>(static_cast<__bf16*>(base) + i));
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

// Units of a thread that are loaded together.
constexpr int kBatch = 2;

// Angles of a workgroup's rows: rows_per_group * pairs of them at most (one per
// thread, or one row's).
constexpr int kAngles = NT > kRopeMaxPairs ? NT : kRopeMaxPairs;

// The units of a head are rotated ones (two per thread and head: units i and
// i + rot/2 of the halves, or, interleaved, two neighbours), then copied ones.
template <bool F32, bool INTER>
__global__ __launch_bounds__(NT) void rope_kernel(RopeParams p) {
  constexpr int N = Unit<F32>::N;
  __shared__ alignas(16) float s_cos[kAngles], s_sin[kAngles];
  const uint32_t half = p.rot / 2;
  const uint32_t rot_units = half / N,
                 units = rot_units + (p.d - p.rot) / N;
  const uint32_t heads = p.heads[0] + p.heads[1], of_row = heads * units;
  const int64_t row0 =
      (int64_t{blockIdx.y} * gridDim.x + blockIdx.x) * p.group_rows;
  if (row0 >= p.rows) return;
  const uint32_t rows = static_cast<uint32_t>(
      min(int64_t{p.group_rows}, p.rows - row0));
  const uint32_t items = rows * of_row;

  struct Item {
    int64_t in, out;
    uint32_t at0, at1, angle;
    int t;
    bool turns;
  };
  auto locate = [&](uint32_t i) {
    Item it;
    const uint32_t r = i / of_row, rest = i - r * of_row;
    const uint32_t h = rest / units, u = rest - h * units;
    it.t = h < uint32_t(p.heads[0]) ? 0 : 1;
    const int64_t row = row0 + r;
    const int64_t head = int64_t{it.t ? h - p.heads[0] : h} * p.d;
    it.in = row * p.x_stride[it.t] + head;
    it.out = row * p.y_stride[it.t] + head;
    it.turns = u < rot_units;
    it.at0 = !it.turns ? p.rot + (u - rot_units) * N
             : INTER   ? 2 * u * N
                       : u * N;
    it.at1 = INTER ? it.at0 + N : it.at0 + half;
    it.angle = r * half + u * N;
    return it;
  };
  Item it[kBatch];
  float x[kBatch][2 * N];
  auto load = [&](uint32_t i0) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (i0 + i * NT >= items) break;
      it[i] = locate(i0 + i * NT);
      Unit<F32>::load(p.x[it[i].t], it[i].in + it[i].at0, x[i]);
      if (it[i].turns)
        Unit<F32>::load(p.x[it[i].t], it[i].in + it[i].at1, x[i] + N);
    }
  };
  load(threadIdx.x);  // in flight while the angles are made
  for (uint32_t i = threadIdx.x; i < rows * half; i += NT) {
    const uint32_t r = i / half, pair = i - r * half;
    float c, s;
    turn_of(p.t.turn[pair], p.positions[p.t.axis[pair] * p.rows + row0 + r], &c,
            &s);
    s_cos[i] = c;
    s_sin[i] = p.inverse ? -s : s;
  }
  lds_barrier();
  for (uint32_t i0 = threadIdx.x; i0 < items; i0 += kBatch * NT) {
    if (i0 != threadIdx.x) load(i0);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      if (i0 + i * NT >= items) break;
      const Item& m = it[i];
      void* y = p.y[m.t];
      if (m.turns) {
        float z[2 * N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float c = s_cos[m.angle + j], s = s_sin[m.angle + j];
          const int a = INTER ? 2 * j : j, e = INTER ? 2 * j + 1 : j + N;
          z[a] = x[i][a] * c - x[i][e] * s;
          z[e] = x[i][e] * c + x[i][a] * s;
        }
        Unit<F32>::store(y, m.out + m.at0, z);
        Unit<F32>::store(y, m.out + m.at1, z + N);
      } else if (p.x[m.t] != y) {
        Unit<F32>::store(y, m.out + m.at0, x[i]);
      }
    }
  }
}

}  // namespace

// Workgroups before one takes more rows.  16384 float32 rows of 20 heads of
// 128, 32 pairs (336 MB): 63.7 us with 4 rows each (4096 workgroups), 69.3 with
// 8; 3001 rows of 16 heads of 64 6.8 us with one each, 10.9 with 16.
constexpr int kGroups = 4096;

hipError_t launch_rope(const RopeParams& params, bool f32,
                       hipStream_t stream) {
  RopeParams p = params;
  // Up to an angle per thread, while there are enough workgroups.
  p.group_rows = 1;
  while (2 * p.group_rows * (p.rot / 2) <= NT &&
         p.rows >= int64_t{2 * p.group_rows} * kGroups)
    p.group_rows *= 2;
  // A launch counts its threads in 32 bits per dimension.
  const int64_t groups = (p.rows + p.group_rows - 1) / p.group_rows;
  const int64_t side = groups < (1 << 22) ? groups : 1 << 22;
  const dim3 g(static_cast<unsigned>(side),
               static_cast<unsigned>((groups + side - 1) / side));
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
