"""Masked co-adaptive MoE layer (MaskCoFT) on AMD Instinct MI355X.

The hot path lives in ``libmaskmoe.so`` (hand-written HIP for gfx950, C ABI in
``include/maskmoe.h``); ``_lib`` is its ctypes binding and ``synth`` the seeded
input generator. Importing the package does not load the library; the first
call into ``_lib`` does, and fails loudly if it has not been built.
"""

from ._lib import (ACT_BF16, ACT_MX4, BF16, CACHE_FIFO, CACHE_LFU, CACHE_LRU, F32, GATE_P, GATE_RENORM,  # noqa: F401
                   GROUP_MAX, GROUP_SUM2, LAYOUT_PACKED, LAYOUT_ROWS, ROUTE_HARD_MASK, ROUTE_PLAIN, ROUTE_SOFT_PRIOR,
                   SCORE_SIGMOID, SCORE_SOFTMAX, LayerDesc, MaskMoEError, PackedMx4Experts, load, make_desc,
                   maskmoe_cache_fetches, maskmoe_experts_backward, maskmoe_experts_backward_workspace_bytes,
                   maskmoe_experts_forward_mx4, maskmoe_experts_forward_train, maskmoe_experts_mx4_workspace_bytes,
                   maskmoe_experts_train_workspace_bytes, maskmoe_gate_backward, maskmoe_gate_forward,
                   maskmoe_layer_forward, maskmoe_layer_workspace_bytes, maskmoe_mx4_dequantize,
                   maskmoe_mx4_pack_experts, maskmoe_mx4_quantize, maskmoe_mx8_dequantize, maskmoe_mx8_quantize,
                   maskmoe_norm_backward, maskmoe_norm_backward_workspace_bytes, maskmoe_norm_forward,
                   maskmoe_pack_expert_weights, maskmoe_route)
