"""B200-native fused W8A8 linear layer: per-token int8 activations x per-channel int8 weights,
int32 accumulation on the tensor cores, dequantization and bias in the GEMM epilogue. Beside it the
4-bit form of the same layer (MXFP4 weights and activations, ``mxfp4``) and a paged cache that keeps
keys and values in int8 or MXFP4 (``kv_cache``).

The compute lives in ``libw8a8_linear.so`` (CUDA, sm_100a; C ABI in ``include/w8a8_linear.h``);
``binding`` is the thin ctypes layer over it. The helper modules ``inputs`` (seeded synthetic
tensors), ``roofline`` (work and byte model) and ``dist`` (multi-rank plumbing) hold none of the
method's arithmetic and do not need the CUDA library: importing them, or this package, maps no
native code. The library is loaded the first time a compute entry point (any name exported by
``binding``, ``mxfp4`` or ``kv_cache``) is touched, and that raises if it has not been built: there is no CPU fallback.
"""
from __future__ import annotations

import importlib

_BINDING_NAMES = (
    "ACT_BF16", "ACT_INT8", "K_MAX", "STATIC_WORKSPACE_BYTES", "W8A8Error", "alloc_workspace", "config_name",
    "force_config", "int8_check_status", "int8_gemm_i32_debug", "int8_linear_fused", "int8_linear_fused_host",
    "int8_linear_fused_static", "int8_linear_workspace_bytes", "int8_linear_workspace_offsets",
    "int8_quantize_act_per_token", "int8_quantize_weight_per_channel", "num_configs",
    "int8_quantize_act_per_token_smooth", "int8_quantize_weight_per_channel_smooth", "int8_linear_fused_smooth",
    "status_string", "int8_linear_workspace_min_bytes", "int8_linear_plan", "int8_sticky_status",
    "debug_set_wait_limit_ns", "debug_set_starve", "debug_set_small_path", "gemm_clock_stamps", "int8_linear_fused_rowmax",
    "int8_quantize_act_per_token_given_absmax",
)
# entry points of the modules next to ``binding``, by module
_MODULE_NAMES = {
    "mxfp4": ("MXFP4_BF16", "MXFP4_CODES", "MXFP4_FP32", "MXFP4_K_MAX", "MXFP4_NUM_CONFIGS", "mxfp4_alloc_workspace", "mxfp4_dequantize", "mxfp4_force_config",
              "mxfp4_linear_fused", "mxfp4_linear_workspace_bytes", "mxfp4_quantize"),
    "kv_cache": ("KV_CACHE_INT8", "KV_CACHE_MAX_DIM", "KV_CACHE_MXFP4", "QuantKVCache", "kv_cache_read", "kv_cache_write"),
}
_MODULE_OF = {name: module for module, names in _MODULE_NAMES.items() for name in names}


def __getattr__(name: str):
    # PEP 562: resolved only when somebody asks for a compute entry point
    if name == "binding" or name in _BINDING_NAMES:
        binding = importlib.import_module(".binding", __name__)
        return binding if name == "binding" else getattr(binding, name)
    if name in _MODULE_NAMES or name in _MODULE_OF:
        module = importlib.import_module("." + _MODULE_OF.get(name, name), __name__)
        if name in _MODULE_NAMES:
            return module
        globals()[name] = getattr(module, name)      # found without this function from now on
        return globals()[name]
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")


def __dir__():
    return sorted(list(globals()) + list(_BINDING_NAMES) + ["binding"] + list(_MODULE_OF) + list(_MODULE_NAMES))
