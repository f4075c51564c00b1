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
  size_t part, H, O;                                            // forward
  size_t x, dyg, xg, row_gate, order, gh, dab, dxr, dgate_part;    // gradient (with part)
  size_t forward_total, backward_total;
};
ExpertsTrainLayout experts_train_layout(int T, int d, int F, int E, int K, int n_shared);
hipError_t launch_experts_train(const ExpertsTrainArgs& a, void* workspace, hipStream_t stream);
hipError_t launch_experts_backward(const ExpertsBwdArgs& a, void* workspace, hipStream_t stream);

// H (bf16 [rows, F]) with its blocks, then O (fp32 expert outputs [rows, d]), on row tiles of kGemmBM (experts.hip).
hipError_t launch_experts_kept(const ExpertArgs& a, const PermBuffers& pb, uint16_t* H, float* O, float* part,
                               const KeptOut& kept, int max_tiles, hipStream_t stream);

// The products of the gradient on rows grouped by expert, in row tiles of kGemmBM (train_products.hip).
struct KeptBwdArgs {
  const uint16_t *w_gate_up, *w_down, *ws_gate_up, *ws_down;
  PermBuffers pb;
  int32_t* order;             // [G] written: the groups, most rows first
  const int8_t* codes;        // [rows, 2F]
  const uint8_t* scales;
  const uint16_t* dy;         // [T, d]
  const uint16_t* x;          // [T, d]
  const uint16_t *dyg, *xg;   // [rows, d] dy and x of each row's token, where gather_rows(F); else null
  uint16_t* gh;               // [rows, F]
  uint16_t* dab;              // [rows, 2F]
  float* dxr;                 // [rows, d]
  float* dgate_part;          // [rows, dgate_parts(F)]
  void *d_w_gate_up, *d_w_down, *d_ws_gate_up, *d_ws_down;
  float* part;                // kTailPartBytes
  int T, d, F, E, G, max_tiles;
};
// Whether the weight gradients read dy and x from rows gathered for them. Reading them by token costs the products 4 %
// (Mixtral-shaped, 8192 tokens, 4810 -> 5020 us; DeepSeek-shaped, 4096 tokens, 735 -> 755), the gathering 80 and 72 us there.
inline bool gather_rows(int F) { return F >= 4096; }
inline int dgate_parts(int F) { return (F + 255) / 256; }
hipError_t launch_experts_backward_products(const KeptBwdArgs& a, hipStream_t stream);

}  // namespace maskmoe
