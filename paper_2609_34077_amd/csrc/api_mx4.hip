// C-ABI entry points of routing by scores, bias and groups, and of MX4 experts: argument validation
// and launches. Nothing is enqueued before every argument has been checked.

#include <math.h>
#include <stdint.h>

#include "gate.hpp"
#include "maskmoe.h"
#include "mx4.hpp"

namespace {

constexpr int kMaxShared = 8;
constexpr int64_t kLim = int64_t{1} << 31;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int hip_status(hipError_t e) { return e == hipSuccess ? MASKMOE_OK : MASKMOE_E_HIP; }

int check_gate(const maskmoe_gate_desc* d) {
  if (!d || d->T < 0 || d->E < 1 || d->E > maskmoe::kGateMaxE || d->K < 1 || d->K > d->E ||
      d->K > maskmoe::kGateMaxK)
    return MASKMOE_E_INVAL;
  if (d->score != MASKMOE_SCORE_SOFTMAX && d->score != MASKMOE_SCORE_SIGMOID) return MASKMOE_E_INVAL;
  if (d->renorm != 0 && d->renorm != 1) return MASKMOE_E_INVAL;
  if (!isfinite(d->scale)) return MASKMOE_E_INVAL;
  if (d->T > 1 << 30) return MASKMOE_E_UNSUPPORTED;   // token numbers and a grid's stride past them fit 32 bits
  return MASKMOE_OK;
}

// Sizes of an MX4 layer; the products need whole 64-column chunks as the bf16 layer does.
int check_mx4(const maskmoe_layer_desc* d) {
  if (!d || d->T < 0 || d->d < 1 || d->F < 1 || d->E < 1 || d->E > 256 || d->K < 1 || d->K > d->E || d->K > 16 ||
      d->n_shared < 0 || d->n_shared > kMaxShared)
    return MASKMOE_E_INVAL;
  if (d->dtype != MASKMOE_BF16 && d->dtype != MASKMOE_F32) return MASKMOE_E_INVAL;
  if (d->dtype != MASKMOE_BF16 || d->d % 64 != 0 || d->F % 64 != 0) return MASKMOE_E_UNSUPPORTED;
  const int64_t rows = static_cast<int64_t>(d->T) * (d->K + d->n_shared);
  if (static_cast<int64_t>(d->T) * d->d >= kLim || rows * d->F >= kLim || int64_t{2} * d->F * d->d >= kLim ||
      rows * d->d >= kLim)
    return MASKMOE_E_UNSUPPORTED;
  if (d->T <= maskmoe::kMx4FewT && rows * d->F >= kLim / 4) return MASKMOE_E_UNSUPPORTED;   // a launch's 2^32 threads
  return MASKMOE_OK;
}

}  // namespace

extern "C" {

int maskmoe_gate_forward(const maskmoe_gate_desc* desc, const float* logits, const uint8_t* mask, const float* prior,
                         const float* bias, int32_t* topk_idx, float* topk_gate, int32_t* load, hipStream_t stream) {
  const int st = check_gate(desc);
  if (st != MASKMOE_OK) return st;
  const maskmoe_gate_desc& d = *desc;
  if (d.n_group < 1 || d.n_group > d.E || d.E % d.n_group != 0 || d.topk_group < 1 || d.topk_group > d.n_group ||
      static_cast<int64_t>(d.topk_group) * (d.E / d.n_group) < d.K)
    return MASKMOE_E_INVAL;
  if (d.group_rule != MASKMOE_GROUP_MAX && d.group_rule != MASKMOE_GROUP_SUM2) return MASKMOE_E_INVAL;
  if (prior)   // in between, neither a key nor its error bound leaves fp32's range
    for (int e = 0; e < d.E; ++e)
      if (!(prior[e] >= 0x1p-100f && prior[e] <= 0x1p100f)) return MASKMOE_E_INVAL;
  if (d.T > 0 && (!logits || !topk_idx || !topk_gate)) return MASKMOE_E_INVAL;
  if (!aligned(logits, 4) || !aligned(bias, 4) || !aligned(topk_idx, 4) || !aligned(topk_gate, 4) || !aligned(load, 4))
    return MASKMOE_E_INVAL;
  maskmoe::GateArgs a{};
  a.logits = logits;
  a.bias = bias;
  a.idx = topk_idx;
  a.gate = topk_gate;
  a.load = load;
  a.T = d.T; a.E = d.E; a.K = d.K; a.score = d.score; a.n_group = d.n_group; a.topk_group = d.topk_group;
  a.group_rule = d.group_rule; a.renorm = d.renorm; a.scale = d.scale;
  a.has_mask = mask != nullptr;
  a.has_prior = prior != nullptr;
  for (int e = 0; e < d.E; ++e) {
    if (mask && mask[e]) a.mask[e >> 5] |= 1u << (e & 31);
    if (prior) a.prior[e] = prior[e];
  }
  return hip_status(maskmoe::launch_gate_forward(a, stream));
}

int maskmoe_gate_backward(const maskmoe_gate_desc* desc, const float* logits, const int32_t* topk_idx,
                          const float* d_gate, float* d_logits, hipStream_t stream) {
  const int st = check_gate(desc);
  if (st != MASKMOE_OK) return st;
  const maskmoe_gate_desc& d = *desc;
  if (d.T == 0) return MASKMOE_OK;
  if (!logits || !topk_idx || !d_gate || !d_logits) return MASKMOE_E_INVAL;
  if (!aligned(logits, 4) || !aligned(topk_idx, 4) || !aligned(d_gate, 4) || !aligned(d_logits, 4) || d_logits == logits)
    return MASKMOE_E_INVAL;
  const maskmoe::GateBwdArgs a{logits, topk_idx, d_gate, d_logits, d.T, d.E, d.K, d.score, d.renorm, d.scale};
  return hip_status(maskmoe::launch_gate_backward(a, stream));
}

static int check_mx4_matrix(int64_t rows, int32_t cols, int32_t dtype, const void* v, const void* codes,
                            const void* scales) {
  if (rows < 0 || cols < 1 || (dtype != MASKMOE_BF16 && dtype != MASKMOE_F32)) return MASKMOE_E_INVAL;
  if (cols % 32 != 0 || rows > (int64_t{1} << 40) / cols) return MASKMOE_E_UNSUPPORTED;
  if (rows > 0 && (!v || !codes || !scales)) return MASKMOE_E_INVAL;
  if (!aligned(v, 16) || !aligned(codes, 16)) return MASKMOE_E_INVAL;
  return MASKMOE_OK;
}

int maskmoe_mx4_quantize(int64_t rows, int32_t cols, int32_t dtype, const void* src, uint8_t* codes, uint8_t* scales,
                         hipStream_t stream) {
  const int st = check_mx4_matrix(rows, cols, dtype, src, codes, scales);
  if (st != MASKMOE_OK || rows == 0) return st;
  return hip_status(maskmoe::launch_mx4_quantize(dtype == MASKMOE_BF16, src, rows, cols, codes, scales, stream));
}

int maskmoe_mx4_dequantize(int64_t rows, int32_t cols, int32_t dtype, const uint8_t* codes, const uint8_t* scales,
                           void* dst, hipStream_t stream) {
  const int st = check_mx4_matrix(rows, cols, dtype, dst, codes, scales);
  if (st != MASKMOE_OK || rows == 0) return st;
  return hip_status(maskmoe::launch_mx4_dequantize(dtype == MASKMOE_BF16, codes, scales, rows, cols, dst, stream));
}

int maskmoe_mx4_packed_bytes(const maskmoe_layer_desc* desc, int32_t n, size_t bytes[4]) {
  if (!desc || !bytes || desc->d < 1 || desc->F < 1 || n < 0) return MASKMOE_E_INVAL;
  if (desc->d % 64 != 0 || desc->F % 64 != 0 || int64_t{2} * desc->F * desc->d >= kLim) return MASKMOE_E_UNSUPPORTED;
  const size_t m = static_cast<size_t>(n);
  bytes[0] = m * maskmoe::mx4_code_bytes(2 * desc->F, desc->d);
  bytes[1] = m * maskmoe::mx4_scale_bytes(2 * desc->F, desc->d);
  bytes[2] = m * maskmoe::mx4_code_bytes(desc->d, desc->F);
  bytes[3] = m * maskmoe::mx4_scale_bytes(desc->d, desc->F);
  return MASKMOE_OK;
}

int maskmoe_mx4_pack_experts(const maskmoe_layer_desc* desc, int32_t n, const maskmoe_mx4_experts* rows,
                             const maskmoe_mx4_experts* packed, hipStream_t stream) {
  size_t bytes[4];
  const int st = maskmoe_mx4_packed_bytes(desc, n, bytes);
  if (st != MASKMOE_OK) return st;
  if (n == 0) return MASKMOE_OK;
  if (!rows || !packed) return MASKMOE_E_INVAL;
  const void* src[] = {rows->gate_up_codes, rows->gate_up_scales, rows->down_codes, rows->down_scales};
  const void* dst[] = {packed->gate_up_codes, packed->gate_up_scales, packed->down_codes, packed->down_scales};
  for (int i = 0; i < 4; ++i)
    if (!src[i] || !dst[i] || src[i] == dst[i] || !aligned(dst[i], 16) || (i % 2 == 0 && !aligned(src[i], 16)))
      return MASKMOE_E_INVAL;
  auto in = [](const void* p) { return static_cast<const uint8_t*>(p); };
  auto out = [](const void* p) { return static_cast<uint8_t*>(const_cast<void*>(p)); };
  const hipError_t err = maskmoe::launch_mx4_pack(in(src[0]), in(src[1]), n, 2 * desc->F, desc->d, true, out(dst[0]),
                                                  out(dst[1]), stream);
  if (err != hipSuccess) return MASKMOE_E_HIP;
  return hip_status(maskmoe::launch_mx4_pack(in(src[2]), in(src[3]), n, desc->d, desc->F, false, out(dst[2]),
                                             out(dst[3]), stream));
}

size_t maskmoe_experts_mx4_workspace_bytes(const maskmoe_layer_desc* desc) {
  if (check_mx4(desc) != MASKMOE_OK) return 0;
  return maskmoe::mx4_layout(desc->T, desc->d, desc->F, desc->E, desc->K, desc->n_shared).total;
}

int maskmoe_experts_forward_mx4(const maskmoe_layer_desc* desc, int32_t act, const void* x, const int32_t* topk_idx,
                                const float* topk_gate, const maskmoe_mx4_experts* w, void* y, void* workspace,
                                size_t workspace_bytes, hipStream_t stream) {
  const int st = check_mx4(desc);
  if (st != MASKMOE_OK) return st;
  if (act != MASKMOE_ACT_BF16 && act != MASKMOE_ACT_MX4) return MASKMOE_E_INVAL;
  if (desc->T == 0) return MASKMOE_OK;
  if (!x || !topk_idx || !topk_gate || !w || !y || x == y) return MASKMOE_E_INVAL;
  const void* ptrs[] = {x, y, w->gate_up_codes, w->gate_up_scales, w->down_codes, w->down_scales};
  for (const void* p : ptrs)
    if (!p || !aligned(p, 16)) return MASKMOE_E_INVAL;
  if (!aligned(topk_idx, 4) || !aligned(topk_gate, 4)) return MASKMOE_E_INVAL;
  if (!workspace || workspace_bytes < maskmoe_experts_mx4_workspace_bytes(desc) || !aligned(workspace, 256))
    return MASKMOE_E_WORKSPACE;
  maskmoe::Mx4Args a;
  a.x = static_cast<const uint16_t*>(x);
  a.idx = topk_idx;
  a.gate = topk_gate;
  a.gu_codes = static_cast<const uint8_t*>(w->gate_up_codes);
  a.gu_scales = static_cast<const uint8_t*>(w->gate_up_scales);
  a.dn_codes = static_cast<const uint8_t*>(w->down_codes);
  a.dn_scales = static_cast<const uint8_t*>(w->down_scales);
  a.y = static_cast<uint16_t*>(y);
  a.T = desc->T; a.d = desc->d; a.F = desc->F; a.E = desc->E; a.K = desc->K; a.n_shared = desc->n_shared;
  a.mx_act = act == MASKMOE_ACT_MX4;
  return hip_status(maskmoe::launch_mx4_experts(a, workspace, stream));
}

}  // extern "C"
