// The 4-bit paged KV cache as its kernels see it: a page's parts and the conversions.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "cw_internal.h"

namespace cw4 {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBs = cw::kBlockSize;
// exponents of the scales that the append writes
constexpr int kMinExp = -100, kMaxExp = 125;

// A page (one block of 16 tokens, one KV head) and the places of its parts, in bytes; the keys' codes
// come first.
template <int D> constexpr int kValues = 8 * D;
template <int D> constexpr int kKeyScales = 16 * D;
template <int D> constexpr int kValueScales = 16 * D + D / 2;
template <int D> constexpr int kPage = 17 * D;

// What a lane holds: D / 16 columns of a token (bf16, codes), and D / 4 codes of a page.
template <int D> struct Piece;
template <> struct Piece<128> {
  typedef u32x4 Bf16;
  typedef uint32_t Code;
  typedef u32x4 Lane;
};
template <> struct Piece<64> {
  typedef u32x2 Bf16;
  typedef uint16_t Code;
  typedef u32x2 Lane;
};

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// The two codes of byte B of `codes` times the scale as bfloat16, exactly (the lower half first). The
// instruction takes the scale's exponent alone: all ones give NaN, zero is 2^-127.
template <int B>
__device__ __forceinline__ uint32_t widen(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B));
}
// The same with a byte that is constant after unrolling.
__device__ __forceinline__ uint32_t widen_at(uint32_t codes, int byte, float scale) {
  return byte == 0 ? widen<0>(codes, scale) : byte == 1 ? widen<1>(codes, scale)
         : byte == 2 ? widen<2>(codes, scale) : widen<3>(codes, scale);
}

// N (4 or 8) values to codes, the first in the lowest bits: nearest, halfway to the even code, 6 at most.
template <int N>
__device__ __forceinline__ uint32_t encode(const float* x, float scale) {
  uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], scale, 1);
  if constexpr (N == 8) {
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], scale, 3);
  }
  return c;
}

}  // namespace cw4
