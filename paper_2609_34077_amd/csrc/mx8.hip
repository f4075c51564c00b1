// Conversion to and from 8-bit blocks (include/maskmoe.h, maskmoe_mx8_quantize, _dequantize). Bound by HBM: every byte
// is read and written once, 16 elements a lane, two lanes a block. bf16, 16384 x 14336 there 144 us and back 143 (5.0 TB/s;
// a copy moves 4.8).

#include "mx8.hpp"

namespace maskmoe {
namespace {

constexpr int kThreads = 256;

// n: elements / 16.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void mx8_quantize_kernel(const void* __restrict__ src, int64_t n,
                                                               int8_t* __restrict__ codes,
                                                               uint8_t* __restrict__ scales) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n; i += step) {
    float v[16];
    load_vec8<BF16>(src, 16 * i, v);
    load_vec8<BF16>(src, 16 * i + 8, v + 8);
    const uint32_t byte = mx8_scale_byte(max_of_2_lanes(max_magnitude<16>(v)));   // n and the step are even: both are here
    uint32_t q[4];
    mx8_encode<16>(v, byte, q);
    reinterpret_cast<u32x4*>(codes)[i] = u32x4{q[0], q[1], q[2], q[3]};
    if ((i & 1) == 0) scales[i >> 1] = static_cast<uint8_t>(byte);
  }
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void mx8_dequantize_kernel(const int8_t* __restrict__ codes,
                                                                 const uint8_t* __restrict__ scales, int64_t n,
                                                                 void* __restrict__ dst) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < n; i += step) {
    const u32x4 q = reinterpret_cast<const u32x4*>(codes)[i];
    const float s = mx8_step(scales[i >> 1]);
    float v[16];
#pragma unroll
    for (int j = 0; j < 4; ++j) mx8_decode4(q[j], s, v + 4 * j);
    store_vec8<BF16>(dst, 16 * i, v);
    store_vec8<BF16>(dst, 16 * i + 8, v + 8);
  }
}

int blocks_for(int64_t n) {
  const int64_t b = (n + kThreads - 1) / kThreads;
  return static_cast<int>(b < 256 * 32 ? b : 256 * 32);
}

}  // namespace

hipError_t launch_mx8_quantize(bool bf16, const void* src, int64_t rows, int cols, int8_t* codes, uint8_t* scales,
                               hipStream_t stream) {
  const int64_t n = rows * cols / 16;
  if (n == 0) return hipSuccess;
  if (bf16) hipLaunchKernelGGL(mx8_quantize_kernel<true>, dim3(blocks_for(n)), dim3(kThreads), 0, stream, src, n, codes, scales);
  else hipLaunchKernelGGL(mx8_quantize_kernel<false>, dim3(blocks_for(n)), dim3(kThreads), 0, stream, src, n, codes, scales);
  return hipGetLastError();
}

hipError_t launch_mx8_dequantize(bool bf16, const int8_t* codes, const uint8_t* scales, int64_t rows, int cols,
                                 void* dst, hipStream_t stream) {
  const int64_t n = rows * cols / 16;
  if (n == 0) return hipSuccess;
  if (bf16) hipLaunchKernelGGL(mx8_dequantize_kernel<true>, dim3(blocks_for(n)), dim3(kThreads), 0, stream, codes, scales, n, dst);
  else hipLaunchKernelGGL(mx8_dequantize_kernel<false>, dim3(blocks_for(n)), dim3(kThreads), 0, stream, codes, scales, n, dst);
  return hipGetLastError();
}

}  // namespace maskmoe
