// Conversion to and from MX4 blocks, and the packing of expert weights (include/maskmoe.h,
// maskmoe_mx4_quantize, _dequantize, _pack_experts). All three are bound by HBM: every byte is read and
// written once, in 16-byte pieces where the type allows.

#include "mx4.hpp"
#include "mx4_block.hpp"

namespace maskmoe {
namespace {

constexpr int kThreads = 256;

// Eight consecutive elements as fp32.
template <bool BF16>
__device__ __forceinline__ void load8(const void* src, int64_t i, float* v) {
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

// Four lanes per block, eight elements each; n: elements / 8.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void mx4_quantize_kernel(const void* __restrict__ src, int64_t n,
                                                               uint32_t* __restrict__ codes,
                                                               uint8_t* __restrict__ scales) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n; i += step) {
    float v[8];
    load8<BF16>(src, 8 * i, v);
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[j]) & 0x7fffffffu);
    // n and the step are multiples of four, so the four lanes of a block are here together
    m = max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0xB1, 0xF, 0xF, true)));
    m = max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0x4E, 0xF, 0xF, true)));
    const uint32_t byte = mx4_scale_byte(m);
    codes[i] = byte == 255 ? 0 : mx4_codes(v, mx4_scale(byte));
    if ((i & 3) == 0) scales[i >> 2] = static_cast<uint8_t>(byte);
  }
}

__device__ __forceinline__ float e2m1_value(uint32_t c) {
  const uint32_t k = c & 7;
  const uint32_t mag = k < 2 ? k : (2 + (k & 1)) << ((k >> 1) - 1);   // in halves
  return (c & 8 ? -0.5f : 0.5f) * static_cast<float>(mag);
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void mx4_dequantize_kernel(const uint32_t* __restrict__ codes,
                                                                 const uint8_t* __restrict__ scales, int64_t n,
                                                                 void* __restrict__ dst) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n; i += step) {
    const uint32_t c = codes[i];
    const float s = mx4_scale(scales[i >> 2]);
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = e2m1_value(c >> (4 * j)) * s;
    if constexpr (BF16) {
      u32x4 q;
#pragma unroll
      for (int j = 0; j < 4; ++j) q[j] = f32x2_to_bf16x2(v[2 * j], v[2 * j + 1]);
      reinterpret_cast<u32x4*>(dst)[i] = q;
    } else {
      f32x4* o = reinterpret_cast<f32x4*>(dst) + 2 * i;
      o[0] = f32x4{v[0], v[1], v[2], v[3]};
      o[1] = f32x4{v[4], v[5], v[6], v[7]};
    }
  }
}

// One wavefront per four steps of a fragment: 4 KiB of codes and 256 bytes of scales.
__global__ __launch_bounds__(kThreads) void mx4_pack_kernel(const uint8_t* __restrict__ codes,
                                                           const uint8_t* __restrict__ scales, int R, int C, int gate_up,
                                                           int64_t units, uint8_t* __restrict__ p_codes,
                                                           uint8_t* __restrict__ p_scales) {
  const int lane = threadIdx.x & 63;
  const int steps = mx4_steps(C), quads = mx4_quads(C), frags = R / 16, blocks = C / kMxBlock;
  const int64_t nw = static_cast<int64_t>(gridDim.x) * (kThreads / kWave);
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * (kThreads / kWave) + (threadIdx.x >> 6); u < units; u += nw) {
    const int q = static_cast<int>(u % quads);
    const int64_t fe = u / quads;                      // fragment over all experts
    const int f = static_cast<int>(fe % frags);
    const int64_t expert = fe / frags;
    const int r16 = gate_up ? (f & 1) * (R / 2) + 16 * (f >> 1) : 16 * f;
    const int64_t row = expert * R + r16 + (lane & 15);
    uint32_t sc = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int s = 4 * q + j;
      if (s >= steps) break;
      const int b = 4 * s + (lane >> 4);
      u32x4 c = {0, 0, 0, 0};
      if (b < blocks) {
        c = *reinterpret_cast<const u32x4*>(codes + (row * blocks + b) * 16);
        sc |= static_cast<uint32_t>(scales[row * blocks + b]) << (8 * j);
      }
      *reinterpret_cast<u32x4*>(p_codes + ((fe * steps + s) * 64 + lane) * 16) = c;
    }
    *reinterpret_cast<uint32_t*>(p_scales + (u * 64 + lane) * 4) = sc;
  }
}

int blocks_for(int64_t n) {
  const int64_t b = (n + kThreads - 1) / kThreads;
  return static_cast<int>(b < 256 * 32 ? b : 256 * 32);
}

}  // namespace

hipError_t launch_mx4_quantize(bool bf16, const void* src, int64_t rows, int cols, uint8_t* codes, uint8_t* scales,
                               hipStream_t stream) {
  const int64_t n = rows * cols / 8;
  if (n == 0) return hipSuccess;
  uint32_t* c = reinterpret_cast<uint32_t*>(codes);
  if (bf16) hipLaunchKernelGGL(mx4_quantize_kernel<true>, dim3(blocks_for(n)), dim3(kThreads), 0, stream, src, n, c, scales);
  else hipLaunchKernelGGL(mx4_quantize_kernel<false>, dim3(blocks_for(n)), dim3(kThreads), 0, stream, src, n, c, scales);
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(bool bf16, const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols,
                                 void* dst, hipStream_t stream) {
  const int64_t n = rows * cols / 8;
  if (n == 0) return hipSuccess;
  const uint32_t* c = reinterpret_cast<const uint32_t*>(codes);
  if (bf16) hipLaunchKernelGGL(mx4_dequantize_kernel<true>, dim3(blocks_for(n)), dim3(kThreads), 0, stream, c, scales, n, dst);
  else hipLaunchKernelGGL(mx4_dequantize_kernel<false>, dim3(blocks_for(n)), dim3(kThreads), 0, stream, c, scales, n, dst);
  return hipGetLastError();
}

hipError_t launch_mx4_pack(const uint8_t* codes, const uint8_t* scales, int n, int R, int C, bool gate_up,
                           uint8_t* p_codes, uint8_t* p_scales, hipStream_t stream) {
  const int64_t units = static_cast<int64_t>(n) * (R / 16) * mx4_quads(C);
  if (units == 0) return hipSuccess;
  hipLaunchKernelGGL(mx4_pack_kernel, dim3(blocks_for(units * 64)), dim3(kThreads), 0, stream, codes, scales, R, C,
                     gate_up ? 1 : 0, units, p_codes, p_scales);
  return hipGetLastError();
}

}  // namespace maskmoe
