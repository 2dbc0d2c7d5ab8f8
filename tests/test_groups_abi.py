"""libogq_groups without a GPU: its symbols, size helpers and refusals, and those of the calls on tensors.  No kernel is launched."""
import ctypes
import os
import re

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2002_11082_amd as ogq
from paper_2002_11082_amd import groups

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x10000  # a fake, aligned device address: never dereferenced on these paths


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(groups.GROUPS_LIB_PATH):
        from paper_2002_11082_amd import build
        build.build()
    return ogq.groups_lib()


def test_every_declared_symbol_is_exported(lib):
    text = open(os.path.join(ROOT, "include", "ogq_groups.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(ogq_[a-z0-9_]+)\s*\(", text)))
    assert len(names) == 12
    for name in names:
        assert hasattr(lib, name), name


def test_size_queries(lib):
    for group in (32, 64, 128):
        p8, p4 = ogq.make_group_params(group, 8), ogq.make_group_params(group, 4)
        assert ogq.ogq_group_codes_bytes(3, group, p8) == 3 * group
        assert ogq.ogq_group_codes_bytes(3, group + 1, p8) == 6 * group
        assert ogq.ogq_group_codes_bytes(3, group + 1, p4) == 3 * group
        assert ogq.ogq_group_exponents_count(3, group + 1, p8) == 6
        assert ogq.ogq_group_codes_bytes(0, 5, p8) == 0 and ogq.ogq_group_codes_bytes(5, 0, p8) == 0
    assert ogq.ogq_group_codes_bytes(1 << 20, 1 << 20, ogq.make_group_params(32, 8)) == 1 << 40
    assert ogq.ogq_group_codes_bytes(3, 5, ogq.make_group_params(16, 8)) == 0
    assert ogq.ogq_group_exponents_count(3, 5, ogq.make_group_params(32, 2)) == 0


def _ref(p):
    return ctypes.byref(p)


def test_refusals(lib):
    p8, p4 = ogq.make_group_params(32, 8), ogq.make_group_params(32, 4)

    def quantize(x=A, stride=64, rows=4, cols=64, dtype=0, p=p8, codes=A, exponents=A):
        return lib.ogq_group_quantize(x, stride, rows, cols, dtype, _ref(p) if p else None, codes, exponents, None)

    assert quantize(p=None) == -1 and quantize(x=0) == -1 and quantize(codes=0) == -1 and quantize(exponents=0) == -1
    assert quantize(p=ogq.make_group_params(48, 8)) == -20 and quantize(p=ogq.make_group_params(0, 8)) == -20
    assert quantize(p=ogq.make_group_params(32, 5)) == -21
    assert quantize(dtype=3) == -22
    assert quantize(x=A + 2) == -6 and quantize(x=A + 1, dtype=1) == -6 and quantize(codes=A + 8) == -6
    assert quantize(rows=1 << 31) == -9 and quantize(cols=1 << 31) == -9 and quantize(rows=1 << 20, cols=1 << 21) == -9
    assert quantize(stride=1 << 60) == -9
    assert quantize(rows=0) == 0 and quantize(cols=0) == 0 and quantize(rows=0, x=0, codes=0, exponents=0) == 0

    def dequantize(codes=A, exponents=A, rows=4, cols=64, p=p8, out=A, stride=64, dtype=0):
        return lib.ogq_group_dequantize(codes, exponents, rows, cols, _ref(p), out, stride, dtype, None)

    assert dequantize(codes=0) == -1 and dequantize(exponents=0) == -1 and dequantize(out=0) == -1
    assert dequantize(stride=63) == -24 and dequantize(codes=A + 4) == -6 and dequantize(out=A + 2) == -6 and dequantize(dtype=9) == -22
    assert dequantize(rows=0, stride=0) == 0

    def forward(x=A, up=None, rows=4, cols=64, dtype=0, act=3, p=p8, y=A, y_stride=64, codes=A, exponents=A, up_codes=None, up_exponents=None):
        return lib.ogq_activation_forward(x, 64, up, 64, rows, cols, dtype, act, _ref(p), y, y_stride, codes, exponents, up_codes, up_exponents, None)

    assert forward(act=4) == -23 and forward(p=p4) == -21 and forward(dtype=4) == -22 and forward(y_stride=0) == -24
    assert forward(x=0) == -1 and forward(y=0) == -1 and forward(codes=0) == -1 and forward(exponents=0) == -1
    assert forward(up=A) == -26 and forward(up=A, up_codes=A) == -26 and forward(up_exponents=A) == -26
    assert forward(up=A + 1, up_codes=A, up_exponents=A) == -6 and forward(up=A, up_codes=A + 1, up_exponents=A) == -6

    def backward(dy=A, codes=A, exponents=A, up_codes=None, up_exponents=None, act=0, p=p8, dx=A, dx_stride=64, dup=None, dup_stride=64):
        return lib.ogq_activation_backward(dy, 64, codes, exponents, up_codes, up_exponents, 4, 64, 0, act, _ref(p), dx, dx_stride, dup, dup_stride, None)

    assert backward(dy=0) == -1 and backward(codes=0) == -1 and backward(dx=0) == -1 and backward(act=7) == -23 and backward(p=p4) == -21
    assert backward(dx_stride=8) == -24 and backward(dup=A) == -26 and backward(up_codes=A, up_exponents=A) == -26
    assert backward(up_codes=A, up_exponents=A, dup=A, dup_stride=8) == -24

    def gradient(dy=A, codes=A, exponents=A, rows=4, outs=8, cols=64, p=p8, accumulate=0, dw=A, stride=64, space=None, size=0, dtype=0):
        return lib.ogq_weight_gradient(dy, 8, dtype, codes, exponents, rows, outs, cols, _ref(p), accumulate, dw, stride, space, size, None)

    assert gradient(dy=0) == -1 and gradient(codes=0) == -1 and gradient(exponents=0) == -1 and gradient(dw=0) == -1
    assert gradient(p=p4) == -21 and gradient(dtype=3) == -22 and gradient(stride=63) == -24 and gradient(dw=A + 2) == -6 and gradient(codes=A + 1) == -6
    assert gradient(outs=1 << 31) == -9
    assert gradient(outs=0) == 0 and gradient(cols=0) == 0 and gradient(rows=0, accumulate=1, dy=0, codes=0, exponents=0) == 0
    need = ogq.ogq_weight_gradient_workspace(100000, 8, 64, ogq.FP32, p8)
    assert need > 0
    assert gradient(rows=100000) == -1 and gradient(rows=100000, space=A, size=need - 1) == -25 and gradient(rows=100000, space=A + 8, size=need) == -6
    assert ogq.ogq_weight_gradient_workspace(100000, 8, 64, 5, p8) == 0 and ogq.ogq_weight_gradient_workspace(100000, 8, 64, 0, p4) == 0

    def matvec(codes=A, exponents=A, outs=8, cols=64, p=p4, x=A, tokens=1, dtype=1, y=A, stride=8):
        return lib.ogq_group_matvec(codes, exponents, outs, cols, _ref(p), x, 64, tokens, dtype, y, stride, None, 0, None)

    assert matvec(codes=0) == -1 and matvec(exponents=0) == -1 and matvec(x=0) == -1 and matvec(y=0) == -1
    assert matvec(p=p8) == -21 and matvec(dtype=3) == -22 and matvec(stride=7) == -24 and matvec(y=A + 1) == -6 and matvec(codes=A + 2) == -6
    assert matvec(tokens=1 << 31) == -9
    assert matvec(tokens=0) == 0 and matvec(outs=0) == 0
    for code in list(range(-26, -19)) + [0, -1, -6, -8, -9]:
        assert ogq.ogq_groups_strerror(code) != "unknown status"
    assert ogq.ogq_groups_strerror(-99) == "unknown status"


def test_missing_library_is_an_error_not_a_fallback(monkeypatch, tmp_path):
    monkeypatch.setattr(groups, "_lib", None)
    monkeypatch.setattr(groups, "GROUPS_LIB_PATH", str(tmp_path / "nope.so"))
    with pytest.raises(ImportError):
        groups.groups_lib()


def _fake(*shape, dtype=torch.bfloat16, device="cuda"):
    with FakeTensorMode():
        return torch.empty(*shape, dtype=dtype, device=device)


def test_tensors_that_the_kernels_could_not_trust_are_refused():
    """All of these are refused before any address is taken."""
    p8, p4 = ogq.make_group_params(32, 8), ogq.make_group_params(32, 4)
    x = _fake(4, 64)
    codes, exponents = _fake(4, 64, dtype=torch.uint8), _fake(4, 2, dtype=torch.uint8)
    codes4 = _fake(4, 32, dtype=torch.uint8)

    def refused(f, error=ValueError):
        with pytest.raises(error):
            f()

    refused(lambda: ogq.ogq_group_quantize(torch.zeros(4, 64), p8))  # host memory
    refused(lambda: ogq.ogq_group_quantize(_fake(64), p8))
    refused(lambda: ogq.ogq_group_quantize(_fake(64, 4).t(), p8))  # values of a row not consecutive
    refused(lambda: ogq.ogq_group_quantize(_fake(4, 64, dtype=torch.float64), p8))
    refused(lambda: ogq.ogq_group_quantize(x, ogq.make_group_params(33, 8)), ogq.OgqError)
    refused(lambda: ogq.ogq_group_quantize(x, ogq.make_group_params(32, 3)), ogq.OgqError)
    refused(lambda: ogq.ogq_group_quantize(x, ogq.make_params(64, 1, ogq.BINGRAD_B)), TypeError)
    refused(lambda: ogq.ogq_group_quantize(None, p8), TypeError)
    refused(lambda: ogq.ogq_group_quantize(x, p8, codes4, exponents))
    refused(lambda: ogq.ogq_group_quantize(x, p8, codes, _fake(4, 2)))
    refused(lambda: ogq.ogq_group_quantize(x, p8, codes, _fake(2, 4, dtype=torch.uint8).t()))
    refused(lambda: ogq.ogq_group_dequantize(codes, exponents, 65, p8, torch.float32))
    refused(lambda: ogq.ogq_group_dequantize(codes, exponents, -1, p8, torch.float32), OverflowError)
    refused(lambda: ogq.ogq_group_dequantize(codes, exponents, 1 << 40, p8, torch.float32))
    refused(lambda: ogq.ogq_group_dequantize(codes, exponents, 64, p8, torch.float64))
    refused(lambda: ogq.ogq_group_dequantize(codes, exponents, 64, p8, torch.float32, _fake(4, 64)))
    refused(lambda: ogq.ogq_group_dequantize(codes, exponents, 64, p4, torch.float32))
    refused(lambda: ogq.ogq_activation_forward(x, ogq.SILU, p8, _fake(4, 63)))
    refused(lambda: ogq.ogq_activation_forward(x, ogq.SILU, p8, _fake(4, 64, dtype=torch.float16)))
    refused(lambda: ogq.ogq_activation_forward(x, ogq.SILU, p8, up_codes=codes))
    refused(lambda: ogq.ogq_activation_forward(x, "silu", p8), TypeError)
    refused(lambda: ogq.ogq_activation_backward(_fake(5, 64), ogq.SILU, codes, exponents, p8))
    refused(lambda: ogq.ogq_activation_backward(x, ogq.SILU, codes, exponents, p8, codes))
    refused(lambda: ogq.ogq_activation_backward(x, ogq.SILU, codes, exponents, p8, dup=x))
    refused(lambda: ogq.ogq_weight_gradient(_fake(3, 8), codes, exponents, 64, p8))
    refused(lambda: ogq.ogq_weight_gradient(_fake(4, 8), codes, exponents, 64, p8, accumulate=True))
    refused(lambda: ogq.ogq_weight_gradient(_fake(4, 8), codes, exponents, 64, p8, _fake(8, 64)))  # dw in fp32
    refused(lambda: ogq.ogq_weight_gradient(_fake(4, 8), codes, exponents, 64, p8, _fake(8, 64, dtype=torch.float32), workspace=torch.zeros(8)))
    refused(lambda: ogq.ogq_group_matvec(codes4, exponents, 64, p4, _fake(1, 63)))
    refused(lambda: ogq.ogq_group_matvec(codes, exponents, 64, p4, _fake(1, 64)))
    refused(lambda: ogq.ogq_group_matvec(codes4, exponents, 64, p4, _fake(1, 64), _fake(1, 4, dtype=torch.float32)))
