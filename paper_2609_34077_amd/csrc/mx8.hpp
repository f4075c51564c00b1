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

// 1 / step where that is a finite number (bytes from 6 on), else its largest power of two: mx8_lift takes the rest.
__device__ __forceinline__ float mx8_inverse_step(uint32_t byte) {
  return __uint_as_float(byte >= 6 ? (260 - byte) << 23 : 254u << 23);
}

// Multiplies the values of blocks below byte 6 (largest magnitude under 2^-121) by what mx8_inverse_step leaves out.
template <int N>
__device__ __forceinline__ void mx8_lift(float* v, uint32_t byte) {
  if (__any(byte < 6)) {
    const float f = __uint_as_float((127 + 6 - min(byte, 6u)) << 23);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] *= f;
  }
}

// v / step as a code in the low byte of the result: nearest integer, ties to even, within -127..127. Adding 1.5 * 2^23
// leaves the rounded integer in the low mantissa bits; v / step is exact (a power of two).
__device__ __forceinline__ uint32_t mx8_code(float v, float inverse_step) {
  constexpr float kMagic = 12582912.0f;
  const float q = __builtin_fmaf(v, inverse_step, kMagic);
  return __float_as_uint(__builtin_amdgcn_fmed3f(q, kMagic - 127.0f, kMagic + 127.0f));
}

// Four values to four codes, the first in the lowest byte.
__device__ __forceinline__ uint32_t mx8_codes4(const float* v, float inverse_step) {
  const uint32_t lo = __builtin_amdgcn_perm(mx8_code(v[1], inverse_step), mx8_code(v[0], inverse_step), 0x0c0c0400u);
  const uint32_t hi = __builtin_amdgcn_perm(mx8_code(v[3], inverse_step), mx8_code(v[2], inverse_step), 0x04000c0cu);
  return lo | hi;
}

// The same for v + rest, |rest| at most half a step of v's last bit: v's distance from its code (exact) and the rest say
// whether the next code is nearer.
__device__ __forceinline__ uint32_t mx8_code(float v, float rest, float inverse_step) {
  constexpr float kMagic = 12582912.0f;
  const float t = v * inverse_step, q = t + kMagic, off = __builtin_fmaf(rest, inverse_step, t - (q - kMagic));
  return __float_as_uint(__builtin_amdgcn_fmed3f(q + ((off + kMagic) - kMagic), kMagic - 127.0f, kMagic + 127.0f));
}

// N values of one block (or more of it in other lanes, `byte` being the whole block's) to N / 4 dwords of codes; 0 for a
// block of byte 255. The values are clobbered.
template <int N>
__device__ __forceinline__ void mx8_encode(float* v, uint32_t byte, uint32_t* codes) {
  mx8_lift<N>(v, byte);
  const float inv = mx8_inverse_step(byte);
#pragma unroll
  for (int i = 0; i < N / 4; ++i) codes[i] = byte == 255 ? 0u : mx8_codes4(v + 4 * i, inv);
}

// The same for v + rest.
template <int N>
__device__ __forceinline__ void mx8_encode(float* v, float* rest, uint32_t byte, uint32_t* codes) {
  mx8_lift<N>(v, byte);
  mx8_lift<N>(rest, byte);
  const float inv = mx8_inverse_step(byte);
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = mx8_code(v[4 * i + j], rest[4 * i + j], inv);
    codes[i] = byte == 255 ? 0u : __builtin_amdgcn_perm(c[1], c[0], 0x0c0c0400u) | __builtin_amdgcn_perm(c[3], c[2], 0x04000c0cu);
  }
}

// The values of four codes (a byte's conversion is one instruction).
__device__ __forceinline__ void mx8_decode4(uint32_t codes, float step, float* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = static_cast<float>(static_cast<int8_t>(codes >> (8 * i))) * step;
}

// Bits of the largest magnitude of N values; a NaN counts as larger than any number.
template <int N>
__device__ __forceinline__ uint32_t max_magnitude(const float* v) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  return m;
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
