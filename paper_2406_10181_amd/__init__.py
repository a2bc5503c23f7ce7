"""MI355X (gfx950) library for the GPU hot path of LSP-Offload: compress S = P^T G Q and
decompress-and-apply W <- W - P S Q^T with (d,r)-sparse ELL projectors (Alg. 1 / Alg. 3, Def. 1),
and the estimation bias of Def. 2 built from the two.  Beside them the operators of a training step that are no plain
matrix products: attention with its backward pass, the norms and the gated residual between two blocks, dropout, the rotation of queries and
keys by position with the norms of their heads, the cross entropy over a vocabulary with its gradients, and AdamW for what has no projector.

This package is a thin binding: it marshals torch device pointers into the C ABI declared in
``include/lsp.h``.  Every step of the path runs in the HIP kernels of ``liblsp_hip.so``; there is
no CPU fallback, and importing the binding fails loudly if the library has not been built.
"""
from .binding import (  # noqa: F401
    LspError, DTYPE_CODE, lib, lib_path,
    lsp_compress, lsp_compress_workspace_bytes, lsp_workspace_bytes,
    lsp_plan_bytes, lsp_plan_build, lsp_plan_build_host, lsp_plan_build_async, lsp_plan_build_workspace_bytes,
    lsp_compress_planned, lsp_compress_planned_workspace_bytes, lsp_compress_planned_static, lsp_static_scratch_bytes,
    lsp_decompress_apply, lsp_compress_planned_grouped, lsp_decompress_apply_grouped, lsp_compress_dense, lsp_compress_dense_workspace_bytes,
    lsp_estimation_bias, lsp_estimation_bias_workspace_bytes,
    lsp_reproject_state, lsp_reproject_state_workspace_bytes, lsp_projector_reorder_host, lsp_projector_reorder,
    lsp_compress_item, lsp_apply_item, compress_items, apply_items, lsp_validate_projector, lsp_strerror, lsp_version,
    torch_dtype_code, lsp_plan_refresh_values, lsp_bias_gradient, lsp_bias_gradient_workspace_bytes, lsp_hbm_probe_read, lsp_hbm_probe_rmw, lsp_hbm_probe_workspace_bytes,
    lsp_dropout, lsp_attention_problem, lsp_attention_gradients, attention_problem, attention_gradients,
    lsp_attention_forward, lsp_attention_forward_workspace_bytes, lsp_attention_backward, lsp_attention_backward_workspace_bytes,
    lsp_residual_norm_problem, lsp_residual_norm_gradients, residual_norm_problem, residual_norm_gradients,
    lsp_residual_norm_forward, lsp_residual_norm_backward, lsp_residual_norm_backward_workspace_bytes,
    lsp_rotary_problem, lsp_rotary_gradients, rotary_problem, rotary_gradients, lsp_rotary_forward, lsp_rotary_backward, lsp_rotary_backward_workspace_bytes,
    lsp_cross_entropy_problem, lsp_cross_entropy_gradients, cross_entropy_problem, cross_entropy_gradients, lsp_cross_entropy_forward,
    lsp_cross_entropy_forward_workspace_bytes, lsp_cross_entropy_backward, lsp_cross_entropy_backward_workspace_bytes,
    lsp_adamw_item, AdamwItems, adamw_items, lsp_adamw,
)
