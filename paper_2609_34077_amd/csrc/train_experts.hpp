// The experts' training pass at a given routing, with the gate / up pre-activations kept in 8-bit blocks: internal
// launchers. Arguments are validated by the C-ABI layer.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "kernels.hpp"

namespace maskmoe {

struct ExpertsTrainArgs {
  const uint16_t* x;          // [T, d]; the gradient: null where x_codes is given
  const int32_t* idx;         // [T, K]
  const float* gate;          // [T, K]
  const uint16_t *w_gate_up, *w_down, *ws_gate_up, *ws_down;
  uint16_t* y;                // forward: [T, d]
  int8_t* codes;              // [rows, 2F]
  uint8_t* scales;            // [rows, 2F / 32]
  int T, d, F, E, K, n_shared;
};
struct ExpertsBwdArgs {
  ExpertsTrainArgs f;         // y unused, codes and scales read
  const int8_t* x_codes;      // [T, d] or null
  const uint8_t* x_scales;    // [T, d / 32]
  const uint16_t* dy;         // [T, d]
  uint16_t* d_x;              // [T, d]
  float* d_gate;              // [T, K] or null
  uint16_t *d_w_gate_up, *d_w_down, *d_ws_gate_up, *d_ws_down;
};

struct ExpertsTrainLayout {   // byte offsets into the workspaces; the grouping is first in both
  size_t idx, gate, offsets, tile_off, wide_off, active, n_active, perm, inv, row_tok, pcount;
  size_t H, O, part;                                            // forward
  size_t dyg, xg, row_gate, order, next, gh, dab, dxr, dgate_part;    // gradient (with part)
  size_t forward_total, backward_total;
};
ExpertsTrainLayout experts_train_layout(int T, int d, int F, int E, int K, int n_shared);
hipError_t launch_experts_train(const ExpertsTrainArgs& a, void* workspace, hipStream_t stream);
hipError_t launch_experts_backward(const ExpertsBwdArgs& a, void* workspace, hipStream_t stream);

// H (bf16 [rows, F]) with its blocks, then O (fp32 expert outputs [rows, d]), on row tiles of kGemmBM (experts.hip).
hipError_t launch_experts_kept(const ExpertArgs& a, const PermBuffers& pb, uint16_t* H, float* O, float* part,
                               const KeptOut& kept, int max_tiles, hipStream_t stream);

// The products of the gradient on rows grouped by expert (backward.hip).
struct KeptBwdArgs {
  const uint16_t *w_gate_up, *w_down, *ws_gate_up, *ws_down;
  PermBuffers pb;
  const int32_t* order;       // [pb.n_active[0]] the groups with rows, most rows first
  int32_t* next;              // [2][8] zeros: tiles that each XCD's workgroups have taken, of each weight gradient
  const int8_t* codes;        // [rows, 2F]
  const uint8_t* scales;
  const uint16_t* dyg;        // [rows, d] dy of each row's token
  const uint16_t* xg;         // [rows, d] x of each row's token
  const float* row_gate;      // [rows]
  uint16_t* gh;               // [rows, F]
  uint16_t* dab;              // [rows, 2F]
  float* dxr;                 // [rows, d]
  float* dgate_part;          // [rows, dgate_parts(F)]
  float* part;                // kTailPartBytes
  void *d_w_gate_up, *d_w_down, *d_ws_gate_up, *d_ws_down;
  int d, F, E, G, max_tiles;
};
inline int dgate_parts(int F) { return (F + 255) / 256; }
hipError_t launch_experts_backward_products(const KeptBwdArgs& a, hipStream_t stream);

}  // namespace maskmoe
