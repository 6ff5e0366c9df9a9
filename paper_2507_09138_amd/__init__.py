"""MI355X-native batched IVF-Flat search, operators around matrices of scores, and layers of the models around them: thin Python
binding over the C ABI of ``hr_ivf.h``, ``hr_scores.h`` and ``hr_layers.h``.

Argument marshalling only; every step runs in the HIP kernels of
``libhr_ivf.so``.  PyTorch supplies device memory and streams.

The names of ``binding``, ``scores`` and ``layers`` are resolved on first use (so that ``python -m
paper_2507_09138_amd.build`` can run before the library exists); using any of them
without a built library raises ImportError.
"""
_NAMES = ["IvfIndex", "HrError", "hr_ivf_load", "hr_ivf_free", "hr_ivf_workspace_bytes",
          "hr_ivf_search", "hr_ivf_search_static", "HR_STATIC_SCRATCH_BYTES", "hr_ivf_coarse", "hr_ivf_scan", "hr_ivf_scan_step", "hr_ivf_scan_step_rows", "hr_ivf_rescore", "hr_ivf_lists_of_rows",
          "hr_ivf_reorder_probes", "reorder_probes", "hr_ivf_list_hits", "hr_ivf_hot_lists", "hr_ivf_refresh_rows", "hr_ivf_set_resident", "hr_ivf_split_probes", "hr_ivf_stats", "hr_ivf_workspace_layout", "hr_ivf_profile_begin",
          "hr_ivf_profile_end", "hr_last_error", "hr_version", "lib", "lib_path", "HR_METRIC_IP",
          "HR_METRIC_L2", "HR_F32", "HR_F16", "HR_BF16", "HR_K_MAX", "HR_NPROBE_MAX", "HR_LOAD_ROW_TABLES"]
# hr_scores.h: operators around a matrix of scores
_SCORES = ["hr_i8_quantize", "hr_i8_workspace_bytes", "hr_i8_product", "hr_i8_linear", "hr_logprobs_workspace_bytes", "hr_logprobs",
           "hr_logprobs_backward", "hr_distill_workspace_bytes", "hr_distill_forward", "hr_distill_backward", "hr_distill_step",
           "quantize_rows", "i8_product", "i8_linear", "Logprobs", "logprobs", "logprobs_backward", "distill_forward",
           "distill_backward", "distill_step", "HR_I8_K_MAX", "HR_LIST_MAX", "HR_ROW_MAX"]
# hr_layers.h: what an encoder or a reader is made of and taught with
_LAYERS = ["hr_layer_norm", "hr_layer_norm_workspace_bytes", "hr_layer_norm_backward", "hr_gated_workspace_bytes", "hr_gated",
           "hr_gated_backward_workspace_bytes", "hr_gated_backward", "hr_adamw", "hr_adamw_moments", "hr_adamw_tensor",
           "LayerNorm", "LayerNormGrads", "layer_norm", "layer_norm_backward", "Gated", "GatedGrads", "gated", "gated_backward", "adamw_state",
           "adamw", "adamw_moments", "HR_SILU", "HR_GELU", "HR_GELU_TANH", "HR_GATED_MAX", "HR_ADAMW_BLOCK"]
__all__ = _NAMES + _SCORES + _LAYERS


def __getattr__(name):
    if name in _NAMES:
        from . import binding
        return getattr(binding, name)
    if name in _SCORES:
        from . import scores
        return getattr(scores, name)
    if name in _LAYERS:
        from . import layers
        return getattr(layers, name)
    raise AttributeError(name)
