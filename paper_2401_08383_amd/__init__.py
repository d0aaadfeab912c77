"""MI355X (gfx950) implementation of the single-GPU hot path of context-coherent MoE inference
with inter-layer expert affinity: the expert layer (gate, dispatch, expert FFN, combine) and the
affinity statistic (co-routing counts, conditional probabilities, placement locality), and the experts' products by themselves:
grouped by expert, with their gradients, with operands in microscaled 4-bit floating point and with weights in 4-bit integers; and routing to many experts, with
the rows of up to 16 experts a token and the gradients of both.

The work is done by hand-written HIP kernels in ``libexflow_moe.so`` (C ABI in
``include/exflow_moe.h``); this package is only the ctypes binding over it.
"""
from .binding import (  # noqa: F401
    EXF_ACT_GELU_ERF,
    EXF_ACT_GELU_TANH,
    EXF_BF16,
    EXF_F32,
    EXF_MX4_BLOCK,
    EXF_SCORE_SIGMOID,
    EXF_SCORE_SOFTMAX,
    ExflowError,
    LIB_PATH,
    Mx4,
    Q4,
    SIGNATURES,
    affinity_histogram,
    affinity_multihop,
    affinity_statistics,
    check_placement,
    comm_volume,
    last_error,
    lib,
    moe_combine,
    moe_combine_backward,
    moe_dispatch,
    moe_dispatch_backward,
    moe_dispatch_static,
    moe_expert_ffn,
    moe_expert_ffn_fused,
    moe_gate_topk,
    moe_grouped_product,
    moe_grouped_product_dw,
    moe_grouped_product_dx,
    moe_grouped_product_mx4,
    moe_grouped_product_q4,
    moe_route,
    moe_route_backward,
    moe_topk_from_logits,
    mx4_dequantize,
    mx4_quantize,
    placement_locality,
    placement_locality_from_counts,
    placement_search,
    q4_dequantize,
    q4_quantize,
    routing_transfers,
    transfer_ratios,
)
