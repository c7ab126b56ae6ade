"""MI355X-native dense GEMM (C = A*B), and products whose rows choose their right operand: thin Python binding of the C-ABI library.

Everything is computed by the HIP kernels in csrc/; this package only loads
libgemm_mi355x.so and marshals arguments.  There is no CPU fallback: if the
library cannot be loaded, calls raise.
"""
from .gemm import (COL_MAJOR, COST_FIXED, COST_HBM, COST_L2, COST_SLAB, ROW_MAJOR, GemmError, config_names, cost_model_scale, force_config, gemm_bf16f32,
                   gemm_f16f16, gemm_f16f32, gemm_f16f32_noalloc, gemm_f32, NOALLOC_SCRATCH_BYTES, last_config, last_kernel, library_path, query_config, set_phase_trace, load_library, shutdown, status_string,
                   tune, tune_clear, tune_save, tune_load, load_tuned_table, TUNED_TABLE, KIND_F32, KIND_F16F32, KIND_F16F16, KIND_BF16F32)
from .routed import (ADAPTERS_MAX_RANK, ELEM_BF16, ELEM_F16, ELEM_F32, KIND_BF16BF16, ROUTE_MAX_EXPERTS, ROUTE_MAX_GROUPS, ROUTE_MAX_TOP_K, SCORE_SIGMOID,
                     SCORE_SOFTMAX, gemm_adapters, gemm_combine, gemm_combine_backward, gemm_grouped, gemm_grouped_wgrad, gemm_route, gemm_route_backward,
                     gemm_route_plan)

__all__ = ["ROW_MAJOR", "COL_MAJOR", "GemmError", "gemm_f32", "gemm_f16f32", "gemm_f16f16", "gemm_bf16f32", "gemm_f16f32_noalloc", "NOALLOC_SCRATCH_BYTES", "force_config",
           "config_names", "query_config", "set_phase_trace", "cost_model_scale", "COST_SLAB", "COST_HBM", "COST_L2", "COST_FIXED", "last_config", "last_kernel", "status_string", "shutdown", "load_library",
           "library_path", "tune", "tune_clear", "tune_save", "tune_load", "load_tuned_table", "TUNED_TABLE", "KIND_F32", "KIND_F16F32", "KIND_F16F16", "KIND_BF16F32",
           "ELEM_F32", "ELEM_F16", "ELEM_BF16", "KIND_BF16BF16", "SCORE_SOFTMAX", "SCORE_SIGMOID", "ROUTE_MAX_EXPERTS", "ROUTE_MAX_GROUPS", "ROUTE_MAX_TOP_K", "ADAPTERS_MAX_RANK", "gemm_route", "gemm_route_backward", "gemm_route_plan", "gemm_grouped", "gemm_grouped_wgrad", "gemm_combine", "gemm_combine_backward", "gemm_adapters"]
