// Routing by scores, balance bias and expert groups: internal launchers (gate.hip). Arguments are
// validated by the C-ABI layer.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace maskmoe {

constexpr int kGateMaxE = 256;
constexpr int kGateMaxK = 16;

struct GateArgs {
  const float* logits;        // [T, E]
  const float* bias;          // [E] or null
  int32_t* idx;               // [T, K]
  float* gate;                // [T, K]
  int32_t* load;              // [E] or null
  int T, E, K, score, n_group, topk_group, group_rule, renorm;
  float scale;
  bool has_mask, has_prior;
  uint32_t mask[kGateMaxE / 32];   // bit e: expert e may be selected
  float prior[kGateMaxE];
};
hipError_t launch_gate_forward(const GateArgs& a, hipStream_t stream);

struct GateBwdArgs {
  const float* logits;        // [T, E]
  const int32_t* idx;         // [T, K]
  const float* d_gate;        // [T, K]
  float* d_logits;            // [T, E]
  int T, E, K, score, renorm;
  float scale;
};
hipError_t launch_gate_backward(const GateBwdArgs& a, hipStream_t stream);

}  // namespace maskmoe
