"""REFLEX variable-K MoE layer for MI355X (gfx950).

The computation lives in ``libreflex.so`` (hand-written HIP kernels behind the C
ABI declared in ``include/reflex.h``).  This package is its Python binding:
``_lib`` mirrors the C entry points one to one, ``layer`` runs the fused layer
from torch tensors (experts in bf16, in e4m3 or in 8-bit integers) and the norms
around it, ``head`` predicts tokens and
confidences of the masked positions, ``trajectory`` runs a whole decode.
Importing the package does not load the library; the first call does, and fails
loudly if it has not been built.
"""
from ._lib import (  # noqa: F401
    ReflexError,
    fp8_scale_shape,
    fp8_weight_scale_shape,
    lib,
    reflex_assign_budget,
    reflex_block_norm,
    reflex_combine,
    reflex_grouped_swiglu,
    reflex_grouped_swiglu_fp8,
    reflex_grouped_swiglu_int8,
    reflex_matmul_fp8,
    reflex_matmul_int8,
    reflex_moe_forward,
    reflex_moe_forward_fp8,
    reflex_moe_forward_int8,
    reflex_permute,
    reflex_permute_workspace_size,
    reflex_quantize_fp8,
    reflex_quantize_fp8_weight,
    reflex_quantize_int8,
    reflex_quantize_int8_weight,
    reflex_router_logits,
    reflex_sample_tokens,
    reflex_sample_workspace_size,
    reflex_select_rows,
    reflex_select_rows_workspace_size,
    reflex_swiglu_fp8_workspace_size,
    reflex_swiglu_int8_workspace_size,
    reflex_swiglu_workspace_size,
    reflex_topk_variable,
    reflex_workspace_fp8_size,
    reflex_workspace_int8_size,
    reflex_workspace_size,
)
