"""Binding of libogq_layers' C ABI (include/ogq_layers.h): rows of a table by tokens, layer norm, a linear layer's product with its bias, activation and residual, the
divergence from a teacher's distribution, and their gradients.  As in groups.py: argument marshalling only, the extension module _marshal for the calls on tensors (values of two
dimensions, CUDA, float32, bfloat16 or float16, consecutive in a row), work enqueued on torch's current stream, no CPU fallback.

Vectors (weight, bias, mean, their gradients) are contiguous float32, tokens and places contiguous int32 or int64.  Outputs and workspaces that are not given are allocated; a
workspace that is given is for one call at a time.

None of the calls is differentiated: a tensor that requires a gradient is read like any other, and the results are not part of its graph.  A program calls the backward pass itself, or from a
torch.autograd.Function.  Outputs of the caller that a call has written get a new version, so that autograd refuses a backward pass that had kept their old values."""
from __future__ import annotations

import ctypes
import os

from . import binding
from .binding import OgqError

LAYERS_LIB_PATH = os.environ.get("OGQ_LAYERS_LIBRARY") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "libogq_layers.so")

INT32, INT64 = 0, 1
IDENTITY = 4

_lib = None


def layers_lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LAYERS_LIB_PATH):
            raise ImportError(
                f"{LAYERS_LIB_PATH} is missing: build it with `python -m paper_2002_11082_amd.build` "
                "(there is no CPU fallback)")
        L = ctypes.CDLL(LAYERS_LIB_PATH)
        sz, vp, u32, i32, f32 = ctypes.c_size_t, ctypes.c_void_p, ctypes.c_uint32, ctypes.c_int, ctypes.c_float
        for name, result, arguments in (
                ("ogq_layer_norm_forward", i32, [vp, sz, sz, sz, u32, vp, vp, f32, vp, sz, vp, vp, vp]),
                ("ogq_layer_norm_backward_workspace", sz, [sz, sz, u32]),
                ("ogq_layer_norm_backward", i32, [vp, sz, vp, sz, sz, sz, u32, vp, vp, vp, vp, sz, vp, vp, i32, vp, sz, vp]),
                ("ogq_linear_workspace", sz, [sz, sz, sz, u32, i32]),
                ("ogq_linear", i32, [vp, sz, vp, sz, i32, sz, sz, sz, u32, vp, u32, vp, sz, vp, sz, vp, sz, vp, sz, vp]),
                ("ogq_linear_backward_workspace", sz, [sz, sz, u32]),
                ("ogq_linear_backward", i32, [vp, sz, sz, sz, u32, u32, vp, sz, vp, sz, vp, i32, vp, sz, vp]),
                ("ogq_embedding_forward", i32, [vp, u32, sz, vp, sz, sz, sz, u32, f32, vp, sz, vp]),
                ("ogq_embedding_gradient_workspace", sz, [sz, sz, sz]),
                ("ogq_embedding_gradient", i32, [vp, u32, sz, vp, sz, sz, sz, u32, f32, i32, vp, sz, vp, sz, vp]),
                ("ogq_distill_workspace", sz, [sz, sz, u32, sz]),
                ("ogq_distill_loss", i32, [vp, sz, sz, sz, u32, vp, u32, vp, sz, f32, vp, vp, vp, sz, vp]),
                ("ogq_distill_gradient", i32, [vp, sz, sz, sz, u32, vp, u32, vp, sz, f32, vp, vp, vp, sz, vp, sz, vp]),
                ("ogq_layers_strerror", ctypes.c_char_p, [i32]),
                ("ogq_layers_last_hip_error", i32, [])):
            f = getattr(L, name)
            f.restype, f.argtypes = result, arguments
        _lib = L
    return _lib


def ogq_layers_strerror(status: int) -> str:
    return layers_lib().ogq_layers_strerror(status).decode()


def _check(status: int) -> None:
    if status != 0:
        raise OgqError(status, ogq_layers_strerror(status))


def ogq_layer_norm_backward_workspace(rows: int, cols: int, dtype: int) -> int:
    """dtype: FP32, BF16 or FP16."""
    return layers_lib().ogq_layer_norm_backward_workspace(rows, cols, dtype)


def ogq_linear_workspace(tokens: int, outs: int, cols: int, dtype: int, transposed: bool = False) -> int:
    """dtype: FP32, BF16 or FP16."""
    return layers_lib().ogq_linear_workspace(tokens, outs, cols, dtype, int(transposed))


def ogq_linear_backward_workspace(tokens: int, outs: int, dtype: int) -> int:
    """dtype: FP32, BF16 or FP16."""
    return layers_lib().ogq_linear_backward_workspace(tokens, outs, dtype)


def ogq_embedding_gradient_workspace(tokens: int, vocab: int, cols: int) -> int:
    return layers_lib().ogq_embedding_gradient_workspace(tokens, vocab, cols)


def ogq_distill_workspace(rows: int, cols: int, dtype: int, top: int) -> int:
    """dtype: FP32, BF16 or FP16."""
    return layers_lib().ogq_distill_workspace(rows, cols, dtype, top)


_marshal = None


def _load_marshal():
    """The extension module that takes tensors, bound to this process's library."""
    global _marshal
    module, L = binding._load_marshal(), layers_lib()
    addresses = [ctypes.cast(f, ctypes.c_void_p).value
                 for f in (L.ogq_layer_norm_forward, L.ogq_layer_norm_backward_workspace, L.ogq_layer_norm_backward, L.ogq_linear_workspace, L.ogq_linear,
                           L.ogq_linear_backward_workspace, L.ogq_linear_backward, L.ogq_embedding_forward, L.ogq_embedding_gradient_workspace,
                           L.ogq_embedding_gradient, L.ogq_distill_workspace, L.ogq_distill_loss, L.ogq_distill_gradient)]
    module.bind_layers(*addresses, _check)
    _marshal = module
    return module


def ogq_layer_norm_forward(x, weight=None, bias=None, eps: float = 1e-5, y=None, mean=None, rstd=None):
    """(x - mean) * rstd * weight + bias for every row.  Returns (y, mean, rstd); the last two are for ogq_layer_norm_backward (and not
    written where there are no columns)."""
    return (_marshal or _load_marshal()).layer_norm_forward(x, weight, bias, eps, y, mean, rstd)


def ogq_layer_norm_backward(dy, x, mean, rstd, weight=None, dx=None, dweight=None, dbias=None, accumulate: bool = False, workspace=None):
    """The gradient of ogq_layer_norm_forward's x from that of its y; with a weight (dx, dweight, dbias), with accumulate the last two added to those that are given.
    dx may be dy.  (The gradient of a bias without a weight is that of ogq_linear_backward(dy).)"""
    return (_marshal or _load_marshal()).layer_norm_backward(dy, x, mean, rstd, weight, dx, dweight, dbias, accumulate, workspace)


def ogq_linear(x, weight, bias=None, activation=None, residual=None, transposed: bool = False, keep: bool = False, y=None, before=None, workspace=None):
    """act(x weight^T + bias) + residual: x [tokens, cols], weight [outs, cols] of x's type, bias float32 [outs].  transposed: weight is [cols, outs], x weight instead (with the
    gradient of a layer's outputs for x and its own weights, the gradient of its inputs).  activation: None, RELU, GELU, GELU_TANH or SILU.  With keep, or before, (y, before), the second one what
    went into the activation.  y may be residual."""
    return (_marshal or _load_marshal()).linear(x, weight, bias, activation, residual, transposed, keep, y, before, workspace)


def ogq_linear_backward(dy, activation=None, before=None, dz=None, dbias=None, accumulate: bool = False, workspace=None):
    """What the backward pass of such a layer begins with: (dz, dbias), dz = dy * act'(before) (dy itself without an activation) and its sums over the tokens, with accumulate added to
    dbias.  The other gradients are ogq_linear(dz, weight, transposed=True) and ogq_weight_gradient(dz, ...).  dz may be dy or before."""
    return (_marshal or _load_marshal()).linear_backward(dy, activation, before, dz, dbias, accumulate, workspace)


def ogq_embedding_forward(tokens, table, scale: float = 1.0, y=None):
    """scale * table[token] for every token; zeros for one that is not in the table."""
    return (_marshal or _load_marshal()).embedding_forward(tokens, table, scale, y)


def ogq_embedding_gradient(tokens, dy, vocab: int, scale: float = 1.0, dtable=None, accumulate: bool = False, workspace=None):
    """The gradient [vocab, cols] (float32) of ogq_embedding_forward's table: scale times the sums of dy's rows of equal tokens; with accumulate, added to dtable."""
    return (_marshal or _load_marshal()).embedding_gradient(tokens, dy, vocab, scale, dtable, accumulate, workspace)


def ogq_distill_loss(logits, places, values, temperature: float = 1.0, row_weight=None, loss=None, workspace=None):
    """The divergence [rows] of softmax(logits / temperature) from the teacher's distribution over `places` [rows, top], softmax(values / temperature), times temperature^2 and the row's
    weight.  A place that is not in the row stands for none."""
    return (_marshal or _load_marshal()).distill_loss(logits, places, values, temperature, row_weight, loss, workspace)


def ogq_distill_gradient(logits, places, values, temperature: float = 1.0, row_weight=None, dlogits=None, loss=None, workspace=None):
    """(loss, dlogits): the same and the gradient of its sum, in one pass over the logits.  dlogits may be logits."""
    return (_marshal or _load_marshal()).distill_gradient(logits, places, values, temperature, row_weight, dlogits, loss, workspace)
