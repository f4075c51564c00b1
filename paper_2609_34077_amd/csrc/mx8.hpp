// Microscaled 8-bit blocks: 32 int8 codes c under one E8M0 scale byte b, standing for c * 2^(b - 133)
// (codes are sixty-fourths of the scale 2^(b - 127)); b = 255 for NaN. Device helpers and internal launchers.
#pragma once

#include "common.hpp"

namespace maskmoe {

constexpr int kMx8Block = 32;

// Scale byte of a block whose largest magnitude has the fp32 bits `amax`: floor(log2(amax)) + 127, which is the
// exponent field (0 for subnormals: 2^-127; 255 for infinities and NaN).
__device__ __forceinline__ uint32_t mx8_scale_byte(uint32_t amax) { return amax >> 23; }

// The value of code 1: 2^(byte - 133), subnormal below byte 7; NaN for 255.
__device__ __forceinline__ float mx8_step(uint32_t byte) {
  const uint32_t bits = byte >= 7 ? (byte - 6) << 23 : 1u << (byte + 16);
  return __uint_as_float(byte == 255 ? 0x7fc00000u : bits);
}

// v / step as a code in the low byte of the result: nearest integer, ties to even, within -127..127. Adding 1.5 * 2^23
// leaves the rounded integer in the low mantissa bits; v / step is exact (a power of two, |v / step| < 128) but where
// it is far below one half.
__device__ __forceinline__ uint32_t mx8_code(float v, uint32_t byte) {
  constexpr float kMagic = 12582912.0f;
  const float q = __builtin_amdgcn_ldexpf(v, 133 - static_cast<int>(byte)) + kMagic;
  return __float_as_uint(__builtin_amdgcn_fmed3f(q, kMagic - 127.0f, kMagic + 127.0f));
}

// Four values to four codes, the first in the lowest byte; 0 for a block of byte 255.
__device__ __forceinline__ uint32_t mx8_codes4(float a, float b, float c, float d, uint32_t byte) {
  const uint32_t lo = __builtin_amdgcn_perm(mx8_code(b, byte), mx8_code(a, byte), 0x0c0c0400u);
  const uint32_t hi = __builtin_amdgcn_perm(mx8_code(d, byte), mx8_code(c, byte), 0x04000c0cu);
  return byte == 255 ? 0u : lo | hi;
}

// Code i (0..3) of a dword.
__device__ __forceinline__ float mx8_code_value(uint32_t codes, int i) {
  return static_cast<float>(static_cast<int32_t>(codes << (24 - 8 * i)) >> 24);
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xF, 0xF, true));
}
// Largest value of the 2 or 4 lanes that share a block.
__device__ __forceinline__ uint32_t max_of_2_lanes(uint32_t m) { return max(m, dpp_u32<0xB1>(m)); }
__device__ __forceinline__ uint32_t max_of_4_lanes(uint32_t m) {
  m = max_of_2_lanes(m);
  return max(m, dpp_u32<0x4E>(m));
}

// Eight consecutive elements as fp32, 16-byte loads.
template <bool BF16>
__device__ __forceinline__ void load_vec8(const void* src, size_t i, float* v) {
  if constexpr (BF16) {
    const u32x4 q = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(src) + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __uint_as_float(q[j] << 16);
      v[2 * j + 1] = __uint_as_float(q[j] & 0xffff0000u);
    }
  } else {
    const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(src) + i);
    const f32x4 a = p[0], b = p[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = a[j], v[4 + j] = b[j];
  }
}

template <bool BF16>
__device__ __forceinline__ void store_vec8(void* dst, size_t i, const float* v) {
  if constexpr (BF16) {
    u32x4 q;
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = f32x2_to_bf16x2(v[2 * j], v[2 * j + 1]);
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(dst) + i) = q;
  } else {
    f32x4* o = reinterpret_cast<f32x4*>(static_cast<float*>(dst) + i);
    o[0] = f32x4{v[0], v[1], v[2], v[3]};
    o[1] = f32x4{v[4], v[5], v[6], v[7]};
  }
}

// codes [rows, cols], scales [rows, cols / 32] of src [rows, cols] (bf16 or fp32), cols % 32 == 0, and back.
hipError_t launch_mx8_quantize(bool bf16, const void* src, int64_t rows, int cols, int8_t* codes, uint8_t* scales,
                               hipStream_t stream);
hipError_t launch_mx8_dequantize(bool bf16, const int8_t* codes, const uint8_t* scales, int64_t rows, int cols,
                                 void* dst, hipStream_t stream);

}  // namespace maskmoe
