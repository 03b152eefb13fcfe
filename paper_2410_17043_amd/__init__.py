"""MI355X-native MoE-layer share (Aurora's data-parallel hot path): HIP kernels behind a C ABI.

Importing this package loads libaurora_moe.so; it raises if the library has not been
built (`python paper_2410_17043_amd/build.py`).  There is no CPU or PyTorch fallback.
"""
import torch  # noqa: F401  (before the library, which then shares torch's HIP runtime: a second one in the process would find no device)

from . import _lib

_lib.load()

from .api import (  # noqa: E402
    F32, BF16, ACT_SILU_MLP, ACT_GELU_MLP, ACT_SWIGLU, TORCH_DTYPE, MoeError, MoeCtx, moe_route, moe_traffic,
    moe_dispatch, moe_dispatch_noalloc, MoeChunkPlan, moe_dispatch_chunks, aurora_chunks, moe_ffn_workspace_bytes, expert_table, moe_expert_ffn, moe_expert_ffn_timed, moe_combine, aurora_order,
    aurora_simulate, colocate_match, aurora_assign, aurora_bottleneck_assign, colocate_hetero_match, aurora_layer_time,
    aurora_colocated_time, Bound, bind_route, bind_traffic, bind_dispatch, bind_dispatch_chunks, bind_expert_ffn,
    bind_combine, moe_diag_mfma_only, moe_diag_copy_1r2w, moe_diag_mfma_run_sum, moe_diag_route_phases, moe_diag_ffn_phases, ffn_phase_marks_len,
    SCORE_SOFTMAX, SCORE_SIGMOID, GROUP_MAX, GROUP_TOP2, gate_rule, moe_fp8_row_bytes, moe_norm_fp8, bind_norm_fp8,
    moe_route_grouped_workspace_bytes, moe_route_grouped, bind_route_grouped, moe_ffn_fp8_workspace_bytes, expert_table_fp8,
    moe_expert_ffn_fp8, bind_expert_ffn_fp8, ROWS_FP8, ROWS_INT8, moe_int8_row_bytes, block_rule, moe_block_norm, bind_block_norm, moe_combine_norm,
    bind_combine_norm, moe_layer_few_workspace_bytes, moe_layer_few, bind_layer_few, moe_quantize_int8, bind_quantize_int8,
    moe_ffn_int8_workspace_bytes, expert_table_int8, moe_expert_ffn_int8, bind_expert_ffn_int8)

__all__ = ["F32", "BF16", "ACT_SILU_MLP", "ACT_GELU_MLP", "ACT_SWIGLU", "TORCH_DTYPE", "MoeError", "MoeCtx",
           "moe_route", "moe_traffic", "moe_dispatch", "moe_dispatch_noalloc", "MoeChunkPlan", "moe_dispatch_chunks", "aurora_chunks", "moe_ffn_workspace_bytes", "expert_table",
           "moe_expert_ffn", "moe_expert_ffn_timed", "moe_combine", "aurora_order", "aurora_simulate", "colocate_match", "aurora_assign", "aurora_bottleneck_assign", "colocate_hetero_match",
           "aurora_layer_time", "aurora_colocated_time", "Bound", "bind_route", "bind_traffic", "bind_dispatch", "bind_dispatch_chunks",
           "bind_expert_ffn", "bind_combine", "moe_diag_mfma_only", "moe_diag_copy_1r2w", "moe_diag_mfma_run_sum",
           "moe_diag_route_phases", "moe_diag_ffn_phases", "ffn_phase_marks_len",
           "SCORE_SOFTMAX", "SCORE_SIGMOID", "GROUP_MAX", "GROUP_TOP2", "gate_rule", "moe_fp8_row_bytes", "moe_norm_fp8", "bind_norm_fp8",
           "moe_route_grouped_workspace_bytes", "moe_route_grouped", "bind_route_grouped", "moe_ffn_fp8_workspace_bytes", "expert_table_fp8",
           "moe_expert_ffn_fp8", "bind_expert_ffn_fp8", "ROWS_FP8", "ROWS_INT8", "moe_int8_row_bytes", "block_rule", "moe_block_norm", "bind_block_norm",
           "moe_combine_norm", "bind_combine_norm", "moe_layer_few_workspace_bytes", "moe_layer_few", "bind_layer_few", "moe_quantize_int8", "bind_quantize_int8",
           "moe_ffn_int8_workspace_bytes", "expert_table_int8", "moe_expert_ffn_int8", "bind_expert_ffn_int8"]
