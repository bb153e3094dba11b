"""MI355X-native sparse weight-delta synchronisation (ROSE, Sec. 4.2): shard_plan, delta_encode,
delta_apply and helpers, and operators at the two ends of a synchronisation (embedding, gradient
norm, 4-bit matrices) and between hidden states and tokens (norms,
distillation, drafted tokens, adapters), implemented in librose_delta.so (HIP, gfx950) and bound with ctypes.

The names of `binding` are served from here on first use, so that `paper_2605_06534_amd.build`
can be run while the library is missing or stale; any other use loads the library and fails
loudly if it is not built (there is no CPU fallback)."""
import importlib

__all__ = ["BF16", "FP32_RNE", "FUSED_ROWS", "REPLICATED", "SPLIT_COLS", "SPLIT_ROWS", "LAYER_FIRST", "LAYER_LAST",
           "Bucket", "Plan", "RoseError", "bucket_check", "bw_probe", "bw_probe_mixed", "bw_probe_lines", "delta_apply", "delta_encode",
           "delta_encode_refresh", "dense_copy", "ENCODE_ARITH", "ENCODE_REFRESH", "PAYLOAD_ARITH", "PAYLOAD_NEW",
           "delta_encode_ex", "delta_encode_static", "delta_apply_ex", "bucket_pack_ex", "bucket_pack", "object_apply",
           "object_bytes", "object_check", "ptr_table", "shard_plan", "workspace", "binding",
           "embedding_lookup", "embedding_grad", "embedding_grad_workspace", "grad_sum_squares", "grad_clip", "grad_clip_norm",
           "grad_workspace", "offset_table", "Mx4", "mx4_quantize", "mx4_dequantize", "mx4_matmul", "mx4_linear",
           "mx4_linear_workspace", "layer_norm", "layer_norm_grad", "layer_norm_grad_workspace", "distill_loss",
           "distill_grad", "distill_loss_grad", "distill_workspace", "draft_verify", "draft_verify_workspace", "Adapters",
           "adapter_linear", "adapter_linear_workspace"]

_names = frozenset(__all__)
_binding = None


def __getattr__(name):
    global _binding
    if name in _names:
        if _binding is None:
            _binding = importlib.import_module(__name__ + ".binding")
        return _binding if name == "binding" else getattr(_binding, name)
    raise AttributeError("module %r has no attribute %r" % (__name__, name))
