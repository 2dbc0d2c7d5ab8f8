"""What autograd is told of the calls of libogq_groups: nothing is differentiated, and what a call has written counts as written."""
import pytest
import torch

import paper_2002_11082_amd as ogq

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
P8, P4 = ogq.make_group_params(32, 8), ogq.make_group_params(32, 4)


def tensors():
    x = torch.randn(4, 64, device=DEV)
    codes, exponents = ogq.ogq_group_quantize(x, P8)
    return x, codes, exponents, *ogq.ogq_group_quantize(x, P4)


def empty(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype, device=DEV)


def calls():
    """(name, outputs, the call that writes them)"""
    x, codes, exponents, codes4, exponents4 = tensors()
    held = lambda: (empty(4, 64, dtype=torch.uint8), empty(4, 2, dtype=torch.uint8))
    c, e = held()
    yield "quantize", (c, e), lambda: ogq.ogq_group_quantize(x, P8, c, e)
    out = empty(4, 64)
    yield "dequantize", (out,), lambda: ogq.ogq_group_dequantize(codes, exponents, 64, P8, torch.float32, out)
    y, fc, fe, uc, ue = empty(4, 64), *held(), *held()
    yield "forward", (y, fc, fe, uc, ue), lambda: ogq.ogq_activation_forward(x, ogq.SILU, P8, x, y, fc, fe, uc, ue)
    dx, dup = empty(4, 64), empty(4, 64)
    yield "backward", (dx, dup), lambda: ogq.ogq_activation_backward(x, ogq.SILU, codes, exponents, P8, codes, exponents, dx, dup)
    dw = empty(64, 64)
    yield "gradient", (dw,), lambda: ogq.ogq_weight_gradient(x, codes, exponents, 64, P8, dw)
    z = empty(4, 4)
    yield "matvec", (z,), lambda: ogq.ogq_group_matvec(codes4, exponents4, 64, P4, x, z)


def test_the_callers_outputs_get_a_new_version():
    for name, outputs, call in calls():
        before = [t._version for t in outputs]
        call()
        assert [t._version for t in outputs] == [v + 1 for v in before], name


def test_autograd_notices_that_a_saved_tensor_was_written():
    for name, outputs, call in calls():
        if not outputs[0].is_floating_point():
            continue
        w = torch.ones_like(outputs[0], requires_grad=True)
        loss = (w * outputs[0]).sum()  # keeps the output's values for w's gradient
        call()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()


def test_outputs_made_in_inference_mode():
    x, codes, exponents, *_ = tensors()
    with torch.inference_mode():
        out = empty(4, 64)
        assert torch.equal(ogq.ogq_group_dequantize(codes, exponents, 64, P8, torch.float32, out), ogq.ogq_group_dequantize(codes, exponents, 64, P8, torch.float32))


def test_results_are_not_part_of_a_graph():
    x = torch.randn(4, 64, device=DEV, requires_grad=True)
    y, *_ = ogq.ogq_activation_forward(x, ogq.SILU, P8)
    assert not y.requires_grad and torch.equal(y, ogq.ogq_activation_forward(x.detach(), ogq.SILU, P8)[0])
