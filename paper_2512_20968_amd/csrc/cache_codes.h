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

}  // namespace dev
}  // namespace mesh_attn
