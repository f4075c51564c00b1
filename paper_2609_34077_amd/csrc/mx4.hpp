// Microscaled 4-bit blocks: internal launchers (mx4.hip) and the layout of packed expert weights
// that the products (mx4_experts.hip) read. Arguments are validated by the C-ABI layer.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "kernels.hpp"

namespace maskmoe {

constexpr int kMxBlock = 32;    // elements that share a scale
constexpr int kMxStep = 128;    // reduction elements of one matrix instruction (16 x 16 x 128)

// codes [rows, cols / 2], scales [rows, cols / 32] of src [rows, cols] (bf16 or fp32), cols % 32 == 0.
hipError_t launch_mx4_quantize(bool bf16, const void* src, int64_t rows, int cols, uint8_t* codes, uint8_t* scales,
                               hipStream_t stream);
hipError_t launch_mx4_dequantize(bool bf16, const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols,
                                 void* dst, hipStream_t stream);

// Packed expert matrix of R rows and C columns (R % 16 == 0, C % 64 == 0), in the operand order of the
// 16 x 16 x 128 matrix instructions. Fragment f holds 16 rows, step s 128 columns (the last one filled up
// with zeros); its 1 KiB at (f * steps + s) is one 16-byte load of a wavefront: lane l the block of row
// l & 15 and columns 128 s + 32 (l >> 4) ... Scales: dword (f * quads + s / 4) * 64 + l, byte s % 4 the
// scale of that block. Fragments of a gate / up matrix alternate: 2q rows 16q .. of W_gate, 2q + 1 the
// same rows of W_up.
inline __host__ __device__ int mx4_steps(int C) { return (C + kMxStep - 1) / kMxStep; }
inline __host__ __device__ int mx4_quads(int C) { return (mx4_steps(C) + 3) / 4; }
inline size_t mx4_code_bytes(int R, int C) { return static_cast<size_t>(R / 16) * mx4_steps(C) * 1024; }
inline size_t mx4_scale_bytes(int R, int C) { return static_cast<size_t>(R / 16) * mx4_quads(C) * 256; }
hipError_t launch_mx4_pack(const uint8_t* codes, const uint8_t* scales, int n, int R, int C, bool gate_up,
                           uint8_t* p_codes, uint8_t* p_scales, hipStream_t stream);

// Experts on packed MX4 weights.
struct Mx4Args {
  const uint16_t* x;       // [T, d] bf16
  const int32_t* idx;      // [T, K]
  const float* gate;       // [T, K]
  const uint8_t *gu_codes, *gu_scales, *dn_codes, *dn_scales;   // E + n_shared experts
  uint16_t* y;             // [T, d] bf16
  int T, d, F, E, K, n_shared;
  bool mx_act;             // activations in MX4 blocks; else bf16
};
struct Mx4Params {
  Mx4Args a;
  const int32_t* idx;   // [T, K + n_shared] experts of every entry; outside [0, G): none
  const float* gate;    // [T, K + n_shared]
  PermBuffers pb;
  uint8_t* xq;       // [T, d / 2] codes
  uint8_t* xs;       // [T, quads of d, 16]: the scale of block b at byte 16 (b / 16) + 4 (b % 4) + b / 4 % 4, so that
                     // dword g of a quad holds the scales of columns 32 g .. of its four steps
  void* h;           // [rows, F] bf16, or codes
  uint8_t* hs;       // [rows, quads of F, 16]
  float* o;          // [rows, d] expert outputs, in as many parts as the down projection's reduction
  int G;             // E + n_shared
};
// Up to kMx4FewT tokens (mx4_few.hip): both products without prepare and permutation; p.o holds kMx4FewSplits x T rows.
constexpr int kMx4FewT = 16, kMx4FewSplits = 32;
// Parts of the down projection's reductions: about four workgroups (64 columns each) a CU, a multiple of 8.
inline int mx4_few_splits(int d) {
  const int s = (1024 / (d / 64) + 7) / 8 * 8;
  return s < 8 ? 8 : s > kMx4FewSplits ? kMx4FewSplits : s;
}
hipError_t launch_mx4_few(const Mx4Params& p, hipStream_t stream);
// Few rows per expert (mx4_batch.hip), the permutation in tiles of kMx4BatchRows; the down projection's reduction in
// `splits` parts, each with its own rows of o.
constexpr int kMx4BatchRows = 64, kMx4BatchSplits = 8, kMx4BatchSplitRows = 8192;
hipError_t launch_mx4_batch(const Mx4Params& p, int max_tiles, int splits, hipStream_t stream);
// Many rows per expert (mx4_tile.hip): both products on tiles of 256 weight rows, the permutation in tiles of
// mx4_tile_rows rows.
constexpr int mx4_tile_rows(bool mx_act) { return mx_act ? 128 : 256; }
hipError_t launch_mx4_wide(const Mx4Params& p, int max_tiles, hipStream_t stream);

struct Mx4Layout {         // byte offsets into the workspace
  size_t idx, gate, offsets, tile_off, active, n_active, perm, inv, row_tok, pcount, xq, xs, h, hs, o, total;
};
Mx4Layout mx4_layout(int T, int d, int F, int E, int K, int n_shared);
hipError_t launch_mx4_experts(const Mx4Args& a, void* workspace, hipStream_t stream);

}  // namespace maskmoe
