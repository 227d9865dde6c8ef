// Angles of rotary positions (gfx950): sine and cosine of a position's turn, a
// 64-bit fraction of a full one (see rope.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mesh_attn {
namespace dev {

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

// The same in float64.
__device__ __forceinline__ void turn_of(uint64_t per, int32_t pos, double* c,
                                        double* s) {
  const uint64_t frac = per * static_cast<uint64_t>(int64_t{pos});
  const uint64_t near = frac + (uint64_t{1} << 61);
  const uint32_t quad = static_cast<uint32_t>(near >> 62);
  const int64_t rest =
      static_cast<int64_t>(frac - (static_cast<uint64_t>(quad) << 62));
  const double t = static_cast<double>(rest) * (6.283185307179586 * 0x1p-64);
  // Taylor: the first terms left out are below 2^-60 of sin and 2^-58 of cos.
  const double z = t * t;
  double sn = fma(z, 1.0 / 355687428096000.0, -1.0 / 1307674368000.0);
  sn = fma(sn, z, 1.0 / 6227020800.0);
  sn = fma(sn, z, -1.0 / 39916800.0);
  sn = fma(sn, z, 1.0 / 362880.0);
  sn = fma(sn, z, -1.0 / 5040.0);
  sn = fma(sn, z, 1.0 / 120.0);
  sn = fma(sn, z, -1.0 / 6.0);
  sn = fma(sn * z, t, t);
  double cs = fma(z, 1.0 / 20922789888000.0, -1.0 / 87178291200.0);
  cs = fma(cs, z, 1.0 / 479001600.0);
  cs = fma(cs, z, -1.0 / 3628800.0);
  cs = fma(cs, z, 1.0 / 40320.0);
  cs = fma(cs, z, -1.0 / 720.0);
  cs = fma(cs, z, 1.0 / 24.0);
  cs = fma(cs, z, -0.5);
  cs = fma(cs, z, 1.0);
  const double a = (quad & 1) ? sn : cs, b = (quad & 1) ? cs : sn;
  *c = (quad == 1 || quad == 2) ? -a : a;
  *s = (quad & 2) ? -b : b;
}

}  // namespace dev
}  // namespace mesh_attn
