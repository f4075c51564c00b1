// Device helpers of MX4 blocks: 32 E2M1 elements (sign, two exponent bits, one mantissa bit: 0, 0.5, 1,
// 1.5, 2, 3, 4, 6) under one E8M0 scale 2^(byte - 127), byte 255 standing for NaN.
#pragma once

#include "common.hpp"

namespace maskmoe {

// Scale byte of a block whose largest magnitude has the fp32 bits `amax`: floor(log2(amax)) - 2, the
// exponent of E2M1's largest value, so that the largest element falls in [4, 8); at least 2^-127.
__device__ __forceinline__ uint32_t mx4_scale_byte(uint32_t amax) {
  const uint32_t e = amax >> 23;
  return e == 255 ? 255 : e > 2 ? e - 2 : 0;
}

// The scale as a float: 2^-127 is subnormal, 255 a NaN; both are mantissa 0x400000.
__device__ __forceinline__ float mx4_scale(uint32_t byte) {
  return __uint_as_float(byte << 23 | (((byte + 1) & 255) < 2 ? 0x400000u : 0u));
}

// Eight fp32 values to eight codes, the first in the lowest bits: v / scale to the nearest element, ties to
// the even mantissa, saturating at 6 (the conversion instruction's rounding, exact on every input tried
// against the definition, subnormals included).
__device__ __forceinline__ uint32_t mx4_codes(const float* v, float scale) {
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], scale, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], scale, 3);
  return r;
}

// Eight codes times their scale as bf16 (exact: two significant bits), a matrix operand register set.
__device__ __forceinline__ u32x4 mx4_to_bf16(uint32_t codes, float scale) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  return r;
}

// A block of 32 bf16 values in one lane (v) to its 16 bytes of codes; returns the scale byte.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t mx4_block_codes(const u32x4 (&v)[4], u32x4& codes) {
  u16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[i][j] & 0x7fff7fffu));
  const uint32_t byte = mx4_scale_byte(static_cast<uint32_t>(m.x > m.y ? m.x : m.y) << 16);
  const float s = mx4_scale(byte);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = v[i][0], b = v[i][1], c = v[i][2], d = v[i][3];
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2_t, a), s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2_t, b), s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2_t, c), s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2_t, d), s, 3);
    codes[i] = byte == 255 ? 0 : r;
  }
  return byte;
}

// Byte of block b's scale in a row of activation scales (Mx4Params::xs).
__device__ __forceinline__ int mx4_scale_at(int b) { return 16 * (b >> 4) + 4 * (b & 3) + (b >> 2 & 3); }

// D = A(16x128) * B(128x16) + C on E2M1 codes with block scales (byte S of sa / sb), fp32 sums.
// Lane l: row (column) l & 15, the block of columns (rows) 32 (l >> 4) ..; result as mfma_16x16x32.
typedef int i32x8 __attribute__((ext_vector_type(8)));
template <int S = 0>
__device__ __forceinline__ f32x4 mfma_mx4(const u32x4& a, const u32x4& b, f32x4 c, uint32_t sa, uint32_t sb) {
  const i32x8 av = {static_cast<int>(a[0]), static_cast<int>(a[1]), static_cast<int>(a[2]), static_cast<int>(a[3]),
                    0, 0, 0, 0};
  const i32x8 bv = {static_cast<int>(b[0]), static_cast<int>(b[1]), static_cast<int>(b[2]), static_cast<int>(b[3]),
                    0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, c, 4, 4, S, static_cast<int>(sa), S,
                                                          static_cast<int>(sb));
}

}  // namespace maskmoe
