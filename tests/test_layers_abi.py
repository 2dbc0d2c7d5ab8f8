"""libogq_layers without a GPU: its symbols, size helpers and refusals, and those of the calls on tensors.  No kernel is launched."""
import os
import re

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2002_11082_amd as ogq
from paper_2002_11082_amd import layers

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x10000  # a fake, aligned device address: never dereferenced on these paths
INF = float("inf")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(layers.LAYERS_LIB_PATH):
        from paper_2002_11082_amd import build
        build.build()
    return ogq.layers_lib()


def test_every_declared_symbol_is_exported(lib):
    text = open(os.path.join(ROOT, "include", "ogq_layers.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(ogq_[a-z0-9_]+)\s*\(", text)))
    assert len(names) == 15
    for name in names:
        assert hasattr(lib, name) and hasattr(ogq, name) or name in ("ogq_layers_last_hip_error",), name


def test_refusals_of_layer_norm(lib):
    def forward(x=A, rows=4, cols=64, dtype=0, weight=A, bias=A, eps=1e-5, y=A, y_stride=64, mean=A, rstd=A, x_stride=64):
        return lib.ogq_layer_norm_forward(x, x_stride, rows, cols, dtype, weight, bias, eps, y, y_stride, mean, rstd, None)

    assert forward(x=0) == -1 and forward(y=0) == -1 and forward(x=A + 2) == -6 and forward(y=A + 1, dtype=1) == -6
    assert forward(weight=A + 2) == -6 and forward(bias=A + 1) == -6 and forward(mean=A + 2) == -6
    assert forward(dtype=3) == -22 and forward(y_stride=63) == -24 and forward(mean=None) == -26 and forward(rstd=None) == -26
    assert forward(eps=-1e-9) == -31 and forward(eps=INF) == -31 and forward(eps=float("nan")) == -31
    assert forward(rows=1 << 31) == -9 and forward(cols=1 << 31) == -9 and forward(rows=1 << 20, cols=1 << 20) == -9 and forward(x_stride=1 << 60) == -9
    assert forward(rows=0, x=0, y=0) == 0 and forward(cols=0, x=0) == 0

    def backward(dy=A, x=A, rows=4, cols=64, dtype=0, weight=A, mean=A, rstd=A, dx=A, dx_stride=64, dw=A, db=A, accumulate=0, space=None, size=0):
        return lib.ogq_layer_norm_backward(dy, 64, x, 64, rows, cols, dtype, weight, mean, rstd, dx, dx_stride, dw, db, accumulate, space, size, None)

    assert backward(dy=0) == -1 and backward(x=0) == -1 and backward(mean=0) == -1 and backward(rstd=0) == -1 and backward(dx=0) == -1
    assert backward(dw=0) == -26 and backward(db=0) == -26 and backward(dx_stride=8) == -24 and backward(dtype=7) == -22 and backward(dw=A + 2) == -6
    need = ogq.ogq_layer_norm_backward_workspace(100000, 64, ogq.FP32)
    assert need > 0 and ogq.ogq_layer_norm_backward_workspace(4, 64, ogq.FP32) == 0 and ogq.ogq_layer_norm_backward_workspace(4, 64, 9) == 0
    assert backward(rows=100000) == -1 and backward(rows=100000, space=A, size=need - 1) == -25 and backward(rows=100000, space=A + 8, size=need) == -6
    assert backward(rows=0, accumulate=1, dy=0) == 0 and backward(rows=0, dw=0, db=0) == 0 and backward(cols=0) == 0


def test_refusals_of_linear_layers(lib):
    def linear(x=A, w=A, transposed=0, tokens=4, outs=8, cols=64, dtype=1, bias=A, act=4, residual=A, y=A, y_stride=8, before=A, before_stride=8, space=None, size=0):
        return lib.ogq_linear(x, 64, w, 64, transposed, tokens, outs, cols, dtype, bias, act, residual, 8, y, y_stride, before, before_stride, space, size, None)

    assert linear(x=0) == -1 and linear(w=0) == -1 and linear(y=0) == -1
    assert linear(x=A + 1) == -6 and linear(w=A + 1) == -6 and linear(bias=A + 2) == -6 and linear(residual=A + 1) == -6 and linear(before=A + 1) == -6
    assert linear(act=5) == -23 and linear(dtype=4) == -22 and linear(y_stride=7) == -24 and linear(before_stride=7) == -24
    assert linear(tokens=1 << 31) == -9 and linear(tokens=1 << 19, outs=1 << 20) == -9
    assert linear(tokens=0) == 0 and linear(outs=0, y=0) == 0
    need = ogq.ogq_linear_workspace(12, 64, 4096, ogq.BF16)
    assert need > 0 and ogq.ogq_linear_workspace(12, 64, 4096, 3) == 0
    assert linear(tokens=12, outs=64, cols=4096, y_stride=64, before_stride=64) == -1
    assert linear(tokens=12, outs=64, cols=4096, y_stride=64, before_stride=64, space=A, size=need - 1) == -25
    assert linear(tokens=12, outs=64, cols=4096, y_stride=64, before_stride=64, space=A + 4, size=need) == -6

    def backward(dy=A, tokens=4, outs=8, dtype=1, act=0, before=A, dz=A, dz_stride=8, dbias=A, accumulate=0, space=None, size=0):
        return lib.ogq_linear_backward(dy, 8, tokens, outs, dtype, act, before, 8, dz, dz_stride, dbias, accumulate, space, size, None)

    assert backward(dy=0) == -1 and backward(before=0) == -1 and backward(dz=0) == -1 and backward(act=9) == -23 and backward(dtype=3) == -22
    assert backward(dz_stride=7) == -24 and backward(dbias=A + 2) == -6
    assert backward(act=4) == -26 and backward(act=4, before=None, dz=None, dbias=None) == -1
    need = ogq.ogq_linear_backward_workspace(1000, 8, ogq.BF16)
    assert need > 0 and ogq.ogq_linear_backward_workspace(16, 8, ogq.BF16) == 0
    assert backward(tokens=1000) == -1 and backward(tokens=1000, space=A, size=need - 1) == -25
    assert backward(outs=0) == 0 and backward(tokens=0, accumulate=1, dy=0) == 0 and backward(tokens=0, dbias=None) == 0


def test_refusals_of_embedding(lib):
    def forward(tokens=A, integer=0, number=4, table=A, vocab=10, cols=8, dtype=0, scale=1.0, y=A, stride=8):
        return lib.ogq_embedding_forward(tokens, integer, number, table, 8, vocab, cols, dtype, scale, y, stride, None)

    assert forward(tokens=0) == -1 and forward(table=0) == -1 and forward(y=0) == -1 and forward(tokens=A + 4, integer=1) == -6 and forward(tokens=A + 2) == -6
    assert forward(integer=2) == -30 and forward(dtype=3) == -22 and forward(scale=INF) == -31 and forward(stride=7) == -24 and forward(number=1 << 31) == -9
    assert forward(number=0, tokens=0) == 0 and forward(cols=0) == 0

    def gradient(tokens=A, integer=0, number=400, dy=A, vocab=10, cols=8, dtype=0, scale=1.0, accumulate=0, out=A, stride=8, space=A, size=1 << 20):
        return lib.ogq_embedding_gradient(tokens, integer, number, dy, 8, vocab, cols, dtype, scale, accumulate, out, stride, space, size, None)

    need = ogq.ogq_embedding_gradient_workspace(400, 10, 8)
    assert need > 0 and ogq.ogq_embedding_gradient_workspace(1 << 30, 10, 1) == 0 and ogq.ogq_embedding_gradient_workspace(200, 10, 8) == 0
    assert gradient(tokens=0) == -1 and gradient(dy=0) == -1 and gradient(out=0) == -1 and gradient(space=None) == -1 and gradient(size=need - 1) == -25 and gradient(space=A + 8) == -6
    assert gradient(integer=2) == -30 and gradient(dtype=3) == -22 and gradient(scale=float("nan")) == -31 and gradient(stride=7) == -24 and gradient(number=1 << 30) == -9
    assert gradient(vocab=0) == 0 and gradient(number=0, accumulate=1, tokens=0, dy=0, space=None, size=0) == 0


def test_refusals_of_distillation(lib):
    def gradient(logits=A, rows=4, cols=64, dtype=1, places=A, integer=1, values=A, top=3, temperature=1.0, weight=A, loss=A, out=A, stride=64, space=None, size=0):
        return lib.ogq_distill_gradient(logits, 64, rows, cols, dtype, places, integer, values, top, temperature, weight, loss, out, stride, space, size, None)

    assert gradient(logits=0) == -1 and gradient(places=0) == -1 and gradient(values=0) == -1 and gradient(out=0) == -1
    assert gradient(places=A + 4) == -6 and gradient(values=A + 2) == -6 and gradient(loss=A + 2) == -6 and gradient(weight=A + 1) == -6 and gradient(logits=A + 1) == -6
    assert gradient(integer=2) == -30 and gradient(dtype=3) == -22 and gradient(stride=63) == -24 and gradient(top=1025) == -9
    for temperature in (0.0, -1.0, INF, float("nan"), 1e-45, 1e30):
        assert gradient(temperature=temperature) == -31
    need = ogq.ogq_distill_workspace(2, 100000, ogq.BF16, 3)
    assert need > 0 and ogq.ogq_distill_workspace(2, 1000, ogq.BF16, 3) == 0
    assert gradient(rows=2, cols=100000, stride=100000) == -1 and gradient(rows=2, cols=100000, stride=100000, space=A, size=need - 1) == -25
    assert gradient(rows=0) == 0 and gradient(cols=0, loss=None) == 0

    def loss(logits=A, places=A, values=A, top=3, out=A):
        return lib.ogq_distill_loss(logits, 64, 4, 64, 1, places, 1, values, top, 1.0, None, out, None, 0, None)

    assert loss(logits=0) == -1 and loss(places=0) == -1 and loss(values=0) == -1 and loss(out=0) == -1
    for code in list(range(-26, -19)) + [0, -1, -6, -8, -9, -30, -31]:
        assert ogq.ogq_layers_strerror(code) != "unknown status"
    assert ogq.ogq_layers_strerror(-99) == "unknown status"


def test_missing_library_is_an_error_not_a_fallback(monkeypatch, tmp_path):
    monkeypatch.setattr(layers, "_lib", None)
    monkeypatch.setattr(layers, "LAYERS_LIB_PATH", str(tmp_path / "nope.so"))
    with pytest.raises(ImportError):
        layers.layers_lib()


def _fake(*shape, dtype=torch.bfloat16, device="cuda"):
    with FakeTensorMode():
        return torch.empty(*shape, dtype=dtype, device=device)


def test_tensors_that_the_kernels_could_not_trust_are_refused():
    """All of these are refused before any address is taken."""
    x, f = _fake(4, 64), lambda *s: _fake(*s, dtype=torch.float32)  # noqa: E731
    ids = _fake(4, 3, dtype=torch.int64)

    def refused(call, error=ValueError):
        with pytest.raises(error):
            call()

    refused(lambda: ogq.ogq_layer_norm_forward(torch.zeros(4, 64)))  # host memory
    refused(lambda: ogq.ogq_layer_norm_forward(_fake(64, 4).t()))
    refused(lambda: ogq.ogq_layer_norm_forward(_fake(4, 64, dtype=torch.float64)))
    refused(lambda: ogq.ogq_layer_norm_forward(x, f(63)))
    refused(lambda: ogq.ogq_layer_norm_forward(x, _fake(64)))  # a weight in fp32
    refused(lambda: ogq.ogq_layer_norm_forward(x, f(64), f(4, 16)))
    refused(lambda: ogq.ogq_layer_norm_forward(x, f(64), eps="small"), TypeError)
    refused(lambda: ogq.ogq_layer_norm_forward(x, y=x, mean=f(5)))
    refused(lambda: ogq.ogq_layer_norm_forward(x, y=_fake(4, 65)))
    refused(lambda: ogq.ogq_layer_norm_backward(x, _fake(5, 64), f(4), f(4)))
    refused(lambda: ogq.ogq_layer_norm_backward(x, x, None, f(4)))
    refused(lambda: ogq.ogq_layer_norm_backward(x, x, f(4), f(4), dweight=f(64)))
    refused(lambda: ogq.ogq_layer_norm_backward(x, x, f(4), f(4), f(64), accumulate=True))
    refused(lambda: ogq.ogq_linear(x, _fake(8, 63)))
    refused(lambda: ogq.ogq_linear(x, _fake(8, 64), transposed=True))
    refused(lambda: ogq.ogq_linear(x, _fake(8, 64, dtype=torch.float16)))
    refused(lambda: ogq.ogq_linear(x, _fake(8, 64), f(7)))
    refused(lambda: ogq.ogq_linear(x, _fake(8, 64), residual=_fake(4, 7), y=_fake(4, 8)))
    refused(lambda: ogq.ogq_linear(x, _fake(8, 64), activation="gelu"), TypeError)
    refused(lambda: ogq.ogq_linear(x, _fake(8, 64), before=f(4, 8), y=_fake(4, 8)))
    refused(lambda: ogq.ogq_linear(x, _fake(8, 64), workspace=torch.zeros(8), y=_fake(4, 8)))
    refused(lambda: ogq.ogq_linear_backward(x, ogq.GELU))
    refused(lambda: ogq.ogq_linear_backward(x, None, x))
    refused(lambda: ogq.ogq_linear_backward(x, None, dz=x))
    refused(lambda: ogq.ogq_linear_backward(x, ogq.GELU, _fake(4, 63)))
    refused(lambda: ogq.ogq_linear_backward(x, accumulate=True))
    refused(lambda: ogq.ogq_embedding_forward(_fake(4, dtype=torch.int16), x))
    refused(lambda: ogq.ogq_embedding_forward(_fake(2, 2, dtype=torch.int64), x))
    refused(lambda: ogq.ogq_embedding_forward(_fake(8, dtype=torch.int64)[::2], x))
    refused(lambda: ogq.ogq_embedding_gradient(_fake(5, dtype=torch.int64), x, 10))
    refused(lambda: ogq.ogq_embedding_gradient(_fake(4, dtype=torch.int64), x, -1), OverflowError)
    refused(lambda: ogq.ogq_embedding_gradient(_fake(4, dtype=torch.int64), x, 10, accumulate=True))
    refused(lambda: ogq.ogq_embedding_gradient(_fake(4, dtype=torch.int64), x, 10, dtable=_fake(10, 64)))
    refused(lambda: ogq.ogq_distill_loss(x, ids, f(4, 4)))
    refused(lambda: ogq.ogq_distill_loss(x, _fake(5, 3, dtype=torch.int64), f(5, 3)))
    refused(lambda: ogq.ogq_distill_loss(x, ids, _fake(4, 3)))
    refused(lambda: ogq.ogq_distill_loss(x, ids, f(4, 3), row_weight=f(5)))
    refused(lambda: ogq.ogq_distill_gradient(x, ids, f(4, 3), dlogits=f(4, 64)))
    refused(lambda: ogq.ogq_distill_gradient(x, f(4, 3), f(4, 3)))
