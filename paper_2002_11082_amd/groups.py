"""Binding of libogq_groups' C ABI (include/ogq_groups.h): tensors held in groups of 8 or 4 bits, and the operators that read
them.  As in binding.py: argument marshalling only, the extension module _marshal for the calls on tensors (two dimensions, CUDA,
float32, bfloat16 or float16, consecutive values in a row), work enqueued on torch's current stream, no CPU fallback.

Codes are uint8 [rows, bytes of a row], exponents uint8 [rows, groups of a row]; see the header for what they stand for.

None of the calls is differentiated: a tensor that requires a gradient is read like any other, and the results are not part of its graph.  A program calls the
backward pass itself (checkpointed_block.py), or from a torch.autograd.Function.  Outputs of the caller that a call has written get a new version, so that autograd
refuses a backward pass that had kept their old values."""
from __future__ import annotations

import ctypes
import os

from . import binding
from .binding import OgqError

GROUPS_LIB_PATH = os.environ.get("OGQ_GROUPS_LIBRARY") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "libogq_groups.so")

FP32, BF16, FP16 = 0, 1, 2
RELU, GELU, GELU_TANH, SILU = 0, 1, 2, 3


class GroupParams(ctypes.Structure):
    """ogq_group_params_t"""
    _fields_ = [("group_size", ctypes.c_uint32), ("bits", ctypes.c_uint32)]


_lib = None


def groups_lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(GROUPS_LIB_PATH):
            raise ImportError(
                f"{GROUPS_LIB_PATH} is missing: build it with `python -m paper_2002_11082_amd.build` "
                "(there is no CPU fallback)")
        L = ctypes.CDLL(GROUPS_LIB_PATH)
        sz, vp, u32, i32 = ctypes.c_size_t, ctypes.c_void_p, ctypes.c_uint32, ctypes.c_int
        pp = ctypes.POINTER(GroupParams)
        for name, result, arguments in (
                ("ogq_group_codes_bytes", sz, [sz, sz, pp]),
                ("ogq_group_exponents_count", sz, [sz, sz, pp]),
                ("ogq_group_quantize", i32, [vp, sz, sz, sz, u32, pp, vp, vp, vp]),
                ("ogq_group_dequantize", i32, [vp, vp, sz, sz, pp, vp, sz, u32, vp]),
                ("ogq_activation_forward", i32, [vp, sz, vp, sz, sz, sz, u32, u32, pp, vp, sz, vp, vp, vp, vp, vp]),
                ("ogq_activation_backward", i32, [vp, sz, vp, vp, vp, vp, sz, sz, u32, u32, pp, vp, sz, vp, sz, vp]),
                ("ogq_weight_gradient_workspace", sz, [sz, sz, sz, u32, pp]),
                ("ogq_weight_gradient", i32, [vp, sz, u32, vp, vp, sz, sz, sz, pp, i32, vp, sz, vp, sz, vp]),
                ("ogq_group_matvec_workspace", sz, [sz, sz, sz, u32, pp]),
                ("ogq_group_matvec", i32, [vp, vp, sz, sz, pp, vp, sz, sz, u32, vp, sz, vp, sz, vp]),
                ("ogq_groups_strerror", ctypes.c_char_p, [i32]),
                ("ogq_groups_last_hip_error", i32, [])):
            f = getattr(L, name)
            f.restype, f.argtypes = result, arguments
        _lib = L
    return _lib


def make_group_params(group_size: int, bits: int = 8) -> GroupParams:
    return GroupParams(group_size, bits)


def ogq_groups_strerror(status: int) -> str:
    return groups_lib().ogq_groups_strerror(status).decode()


def _check(status: int) -> None:
    if status != 0:
        raise OgqError(status, ogq_groups_strerror(status))


def ogq_group_codes_bytes(rows: int, cols: int, params: GroupParams) -> int:
    return groups_lib().ogq_group_codes_bytes(rows, cols, ctypes.byref(params))


def ogq_group_exponents_count(rows: int, cols: int, params: GroupParams) -> int:
    return groups_lib().ogq_group_exponents_count(rows, cols, ctypes.byref(params))


def ogq_weight_gradient_workspace(rows: int, outs: int, cols: int, dtype: int, params: GroupParams) -> int:
    """dtype: FP32, BF16 or FP16."""
    return groups_lib().ogq_weight_gradient_workspace(rows, outs, cols, dtype, ctypes.byref(params))


def ogq_group_matvec_workspace(tokens: int, outs: int, cols: int, dtype: int, params: GroupParams) -> int:
    """dtype: FP32, BF16 or FP16."""
    return groups_lib().ogq_group_matvec_workspace(tokens, outs, cols, dtype, ctypes.byref(params))


_marshal = None


def _load_marshal():
    """The extension module that takes tensors, bound to this process's library."""
    global _marshal
    module, L = binding._load_marshal(), groups_lib()
    addresses = [ctypes.cast(f, ctypes.c_void_p).value
                 for f in (L.ogq_group_codes_bytes, L.ogq_group_exponents_count, L.ogq_group_quantize, L.ogq_group_dequantize,
                           L.ogq_activation_forward, L.ogq_activation_backward, L.ogq_weight_gradient_workspace,
                           L.ogq_weight_gradient, L.ogq_group_matvec_workspace, L.ogq_group_matvec)]
    module.bind_groups(*addresses, _check, GroupParams)
    _marshal = module
    return module


def ogq_group_quantize(x, params: GroupParams, codes=None, exponents=None):
    """x [rows, cols] into groups.  Returns (codes, exponents)."""
    return (_marshal or _load_marshal()).group_quantize(x, params, codes, exponents)


def ogq_group_dequantize(codes, exponents, cols: int, params: GroupParams, dtype, out=None):
    """What codes and exponents stand for, as [rows, cols] in `dtype` (a torch dtype)."""
    return (_marshal or _load_marshal()).group_dequantize(codes, exponents, cols, params, dtype, out)


def ogq_activation_forward(x, activation: int, params: GroupParams, up=None, y=None, codes=None, exponents=None, up_codes=None,
                           up_exponents=None):
    """y = act(x), or act(x) * up; x (and up) are left in 8 bits for the backward pass, ogq_activation_backward (y is in no graph of autograd's).
    activation: RELU, GELU, GELU_TANH or SILU.  Returns (y, codes, exponents), with up also (up_codes, up_exponents) behind them."""
    return (_marshal or _load_marshal()).activation_forward(x, activation, params, up, y, codes, exponents, up_codes, up_exponents)


def ogq_activation_backward(dy, activation: int, codes, exponents, params: GroupParams, up_codes=None, up_exponents=None, dx=None,
                            dup=None):
    """The gradient of ogq_activation_forward's x from that of its y and what it left; with up_codes and up_exponents
    (dx, dup), the gradient of up too."""
    return (_marshal or _load_marshal()).activation_backward(dy, activation, codes, exponents, params, up_codes, up_exponents, dx, dup)


def ogq_weight_gradient(dy, codes, exponents, cols: int, params: GroupParams, dw=None, accumulate: bool = False, workspace=None):
    """The gradient [outs, cols] (float32) of a linear layer's weights: dy [rows, outs] transposed times the checkpointed inputs
    [rows, cols]; with accumulate, added to dw."""
    return (_marshal or _load_marshal()).weight_gradient(dy, codes, exponents, cols, params, dw, accumulate, workspace)


def ogq_group_matvec(codes, exponents, cols: int, params: GroupParams, x, y=None, workspace=None):
    """x [tokens, cols] times the transpose of the weights [outs, cols] held in 4 bits: [tokens, outs] in x's type."""
    return (_marshal or _load_marshal()).group_matvec(codes, exponents, cols, params, x, y, workspace)
