// Internal launchers of the root-mean-square norm (norm.hip). Arguments are validated by the C-ABI layer.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace maskmoe {

constexpr int kNormMaxD = 32768;   // a row stays in the registers of one workgroup

struct NormArgs {
  const void* x;          // [T, d]
  const void* residual;   // [T, d] or null
  const void* weight;     // [d]
  void* hidden;           // [T, d] x + residual, or null
  void* y;                // [T, d] or null
  int8_t* codes;          // [T, d] or null (d % 32 == 0)
  uint8_t* scales;        // [T, d / 32]
  int T, d;
  float eps;
  bool bf16;
};
hipError_t launch_norm_forward(const NormArgs& a, hipStream_t stream);

struct NormBwdArgs {
  const void* hidden;     // [T, d] what the norm read
  const void* weight;     // [d]
  const void* dy;         // [T, d]
  const void* d_hidden;   // [T, d] or null
  void* d_x;              // [T, d]
  float* d_weight;        // [d] or null
  float* part;            // workspace [norm_backward_parts, d] when d_weight is given
  int T, d;
  float eps;
  bool bf16;
};
int norm_backward_parts(int T, int d);
hipError_t launch_norm_backward(const NormBwdArgs& a, hipStream_t stream);

}  // namespace maskmoe
