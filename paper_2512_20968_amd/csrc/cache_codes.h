// Device helpers of the 4-bit cache: E2M1 codes, scales and addresses (gfx950).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache.h"

namespace mesh_attn {
namespace dev {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// c and the sum of eight bf16, exact products: what a second product's operand adds
// up to.
__device__ __forceinline__ float add_eight(const bf16x8& x, float c) {
  const bf16x2 one = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16x2 y = {x[2 * i], x[2 * i + 1]};
    c = __builtin_amdgcn_fdot2_f32_bf16(y, one, c, false);
  }
  return c;
}

constexpr uint32_t kScaleNaN = 255;  // scale code of a group of NaN

// The scale 2^(code - 127) as a float: the code is its exponent field.
__device__ __forceinline__ float scale_of(uint32_t code) {
  return __uint_as_float(code << 23);
}

// The two values of byte `Byte` of w, times the scale.  Values and scales are
// powers of two apart, so the products are exact in bf16.
template <int Byte>
__device__ __forceinline__ bf16x2 dequant2(uint32_t w, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, Byte);
}

// The eight values of w in order, as the registers of an MFMA operand.
__device__ __forceinline__ bf16x8 dequant8(uint32_t w, float scale) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, dequant2<0>(w, scale));
  r[1] = __builtin_bit_cast(uint32_t, dequant2<1>(w, scale));
  r[2] = __builtin_bit_cast(uint32_t, dequant2<2>(w, scale));
  r[3] = __builtin_bit_cast(uint32_t, dequant2<3>(w, scale));
  return __builtin_bit_cast(bf16x8, r);
}

// Byte offsets inside a (page, KV head) block of page size 2^lg.
template <int D>
struct Block {
  static constexpr int kGroups = D / 32;
  // K codes of token t; V codes of the token's eight-token run, then of column
  // n (its D/16 dims) and of the token; scales.
  __device__ static int k_codes(int, int t) { return t * (D / 2); }
  __device__ static int v_codes(int lg, int t, int n) {
    return ((D / 2) << lg) + (t >> 3) * (4 * D) + n * (D / 4) +
           (t & 7) * (D / 32);
  }
  __device__ static int k_scale(int lg, int t, int g) {
    return (D << lg) + t * kGroups + g;
  }
  __device__ static int v_scale(int lg, int t, int g) {
    return ((D + kGroups) << lg) + (g << lg) + t;
  }
};

// Codes of 8 values and their group's scale code.
struct Quant {
  uint32_t codes, scale;
};

// Of the values of four neighbouring lanes, a group, this lane's.
__device__ __forceinline__ Quant quantize8(float (&x)[8]) {
  uint32_t top = 0;  // largest magnitude, as float bits (NaN above infinity)
#pragma unroll
  for (int i = 0; i < 8; ++i)
    top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
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

// Dims 8 chunk .. of K and V of token t into its (page, KV head) block.
template <int D>
__device__ __forceinline__ void store_quants(uint8_t* blk, int lg, int t,
                                             int chunk, const Quant& k,
                                             const Quant& v) {
  using B = Block<D>;
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

}  // namespace dev
}  // namespace mesh_attn
