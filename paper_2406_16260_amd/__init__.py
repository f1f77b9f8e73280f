"""dsattn: Dual-scope temporal self-attention (Video-Infinity, arXiv 2406.16260, Section 4.2)
as hand-written HIP kernels for gfx950 behind a C ABI (include/dsattn.h).

`binding` mirrors the C entry points; `synth` holds the seeded synthetic workloads;
`build` compiles libdsattn.so in-tree.  Attribute access is lazy so that importing the
package (e.g. for `synth`) does not require the built library.
"""
import importlib

_BINDING_NAMES = (
    "dsattn_plan", "dsattn_plan_destroy", "dsattn_plan_ctx_max", "dsattn_plan_ctx_indices",
    "dsattn_plan_launch_info", "dsattn_gather_context", "dsattn_forward", "dsattn_forward_ctx",
    "dsattn_copy_probe", "dsattn_strerror", "dsattn_last_error", "dsattn_groupnorm",
    "dsattn_groupnorm_workspace", "Plan", "DsattnError",
    "dsattn_groupnorm_static", "dsattn_groupnorm_static_max_bytes", "dsattn_temporal_conv",
    "dsattn_temporal_conv_info", "dsattn_linear", "dsattn_linear_info", "dsattn_temporal_layer",
    "dsattn_temporal_layer_workspace", "dsattn_rmsnorm", "dsattn_linear_act", "dsattn_linear_act_info",
    "dsattn_sink_workspace", "dsattn_sink_forward", "dsattn_sink_forward_info",
    "dsattn_layernorm", "dsattn_layernorm_backward_workspace", "dsattn_layernorm_backward",
    "dsattn_gated_scan_workspace", "dsattn_gated_scan", "dsattn_gated_scan_backward",
    "dsattn_linear_act_backward_workspace", "dsattn_linear_act_backward",
    "DSATTN_SCAN_SUM", "DSATTN_SCAN_MEAN", "DSATTN_SCAN_NORM", "DSATTN_SCAN_FRAMES",
    "DSATTN_F32", "DSATTN_BF16", "DSATTN_E4M3", "DSATTN_ACT_NONE", "DSATTN_ACT_RELU", "DSATTN_ACT_GELU",
    "DSATTN_ACT_GELU_TANH", "DSATTN_ACT_SILU", "DSATTN_FLAG_FORCE_GENERIC", "DSATTN_FLAG_SLIDING_WINDOW",
    "DSATTN_FLAG_DEDUP_GLOBAL", "DSATTN_FLAG_FP32_SUMS",
)


def __getattr__(name):
    if name in _BINDING_NAMES:
        return getattr(importlib.import_module(".binding", __name__), name)
    if name in ("binding", "synth", "build"):
        return importlib.import_module("." + name, __name__)
    raise AttributeError(name)
