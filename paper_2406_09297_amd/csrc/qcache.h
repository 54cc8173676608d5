// Device side of the 4-bit cache (layout in serve.h): places inside a record,
// quantisation of a row's block and the values of codes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "serve.h"
#include "tile.h"

namespace mlkv {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <int D>
struct QTile {
  static constexpr int KK = D / 32;
  static constexpr int kBytes = kQTileBytes(D);
  static constexpr int kVCodes = 16 * D, kKExps = 32 * D, kVExps = 33 * D;

  // Byte offsets of token u (0 .. 31) of a record: the dword of key channels
  // 8 c .. 8 c + 7, the exponents of key and value channels 32 b .. 32 b + 31.
  __device__ __forceinline__ static int k_dword(int u, int c) {
    const int i = ((u >> 2) & 1) * KK + (c >> 2);
    const int lane = (c & 3) * 16 + ((u >> 3) << 2) + (u & 3);
    return (i >> 2) * 1024 + lane * 16 + (i & 3) * 4;
  }
  __device__ __forceinline__ static int k_exp(int u, int b) {
    return kKExps + (((u >> 3) << 2) + (u & 3)) * 2 * KK + ((u >> 2) & 1) * KK + b;
  }
  __device__ __forceinline__ static int v_exp(int u, int b) {
    return kVExps + (u >> 3) * 8 * KK + b * 8 + (u & 7);
  }
};

__device__ __forceinline__ float exp_scale(uint32_t byte) {
  return __builtin_bit_cast(float, byte << 23);
}

// The exponent byte of a block whose largest magnitude has bf16 pattern `top`:
// the least 2^e with top < 7 2^e (adding a quarter of a binade carries where
// the magnitude passes 1.75 of its power of two), so that the largest value
// becomes 4 or 6 steps and none is more than half a step of its place off, save
// those from 7 2^125 on, which become 6 steps of 2^125.
__device__ __forceinline__ int block_exp(int top) {
  if (top >= 0x7F80) return kQNaN;
  const int e = ((top + 0x20) >> 7) - 2;
  return e < kQMinExp ? kQMinExp : e > kQMaxExp ? kQMaxExp : e;
}

// Eight values (bf16) of a block to their codes, value i in nibble i.  The
// conversion rounds to nearest, ties to the even code.  A block that is not
// finite has codes of 0: its scale alone makes it NaN.
__device__ __forceinline__ uint32_t quantise8(u16x8 x, int exp_byte) {
  if (exp_byte == kQNaN) return 0;
  const float scale = exp_scale(exp_byte);
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    f[i] = __builtin_bit_cast(float, static_cast<uint32_t>(x[i]) << 16);
  uint32_t d = 0;
  d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, f[0], f[1], scale, 0);
  d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, f[2], f[3], scale, 1);
  d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, f[4], f[5], scale, 2);
  d = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(d, f[6], f[7], scale, 3);
  return d;
}

// The eight values codes times 2^e stand for, exactly (bf16 holds every one);
// the conversion reads only the scale's exponent bits, and makes NaN of 255.
__device__ __forceinline__ u16x8 dequantise8(uint32_t codes, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  u32x4 d;
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  const bf16x2 e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  d[0] = __builtin_bit_cast(uint32_t, a);
  d[1] = __builtin_bit_cast(uint32_t, b);
  d[2] = __builtin_bit_cast(uint32_t, c);
  d[3] = __builtin_bit_cast(uint32_t, e);
  return __builtin_bit_cast(u16x8, d);
}

}  // namespace mlkv
