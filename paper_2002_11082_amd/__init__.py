"""Per-bucket optimal gradient quantization (BinGrad-b / ORQ, arXiv 2002.11082) on MI355X.

The product is libogq.so (HIP kernels behind the C ABI declared in include/ogq.h); this package
is the thin Python binding plus the seeded synthetic-input generators used by tests and bench.  Beside it libogq_groups.so
(include/ogq_groups.h, groups.py): activations held in 8 bits until the backward pass, weights held in 4 bits for serving; and libogq_layers.so
(include/ogq_layers.h, layers.py): embedding, layer norm, linear layers and distillation, forward and backward.
"""
from .binding import (BINGRAD_B, BINGRAD_PB, EVEN, LINEAR, MAX_WORKERS, ORQ, ORQ_PAPER, SCALED_SIGN, OgqError, Params, lib, make_params, ogq_codes_bytes,
                      ogq_dequantize_average, ogq_dequantize_average_raw, ogq_levels_count, ogq_levels_per_bucket,
                      ogq_num_buckets,
                      ogq_probe_copy, ogq_probe_read, ogq_quantize, ogq_quantize_raw, ogq_strerror)
from .groups import (BF16, FP16, FP32, GELU, GELU_TANH, RELU, SILU, GroupParams, groups_lib, make_group_params, ogq_activation_backward,
                     ogq_activation_forward, ogq_group_codes_bytes, ogq_group_dequantize, ogq_group_exponents_count,
                     ogq_group_matvec, ogq_group_matvec_workspace, ogq_group_quantize, ogq_groups_strerror, ogq_weight_gradient,
                     ogq_weight_gradient_workspace)
from .layers import (IDENTITY, INT32, INT64, layers_lib, ogq_distill_gradient, ogq_distill_loss, ogq_distill_workspace, ogq_embedding_forward,
                     ogq_embedding_gradient, ogq_embedding_gradient_workspace, ogq_layer_norm_backward, ogq_layer_norm_backward_workspace,
                     ogq_layer_norm_forward, ogq_layers_strerror, ogq_linear, ogq_linear_backward, ogq_linear_backward_workspace,
                     ogq_linear_workspace)

__all__ = [
    "BINGRAD_B", "BINGRAD_PB", "ORQ", "ORQ_PAPER", "SCALED_SIGN", "EVEN", "LINEAR", "MAX_WORKERS", "ogq_levels_per_bucket", "OgqError", "Params", "lib", "make_params", "ogq_codes_bytes",
    "ogq_dequantize_average", "ogq_dequantize_average_raw", "ogq_levels_count", "ogq_num_buckets", "ogq_probe_copy",
    "ogq_probe_read", "ogq_quantize", "ogq_quantize_raw", "ogq_strerror",
    "FP32", "BF16", "FP16", "RELU", "GELU", "GELU_TANH", "SILU", "GroupParams", "groups_lib", "make_group_params", "ogq_activation_backward",
    "ogq_activation_forward", "ogq_group_codes_bytes", "ogq_group_dequantize", "ogq_group_exponents_count", "ogq_group_matvec",
    "ogq_group_matvec_workspace", "ogq_group_quantize", "ogq_groups_strerror", "ogq_weight_gradient", "ogq_weight_gradient_workspace",
    "IDENTITY", "INT32", "INT64", "layers_lib", "ogq_distill_gradient", "ogq_distill_loss", "ogq_distill_workspace", "ogq_embedding_forward",
    "ogq_embedding_gradient", "ogq_embedding_gradient_workspace", "ogq_layer_norm_backward", "ogq_layer_norm_backward_workspace",
    "ogq_layer_norm_forward", "ogq_layers_strerror", "ogq_linear", "ogq_linear_backward", "ogq_linear_backward_workspace",
    "ogq_linear_workspace",
]
