"""Activations of libogq_groups over all of their range, on the GPU against the definitions in 64 bits, by bounds that are relative to the results: the tails
where an activation is a small difference or a small quotient are held to as many bits as the rest.

In 32 bits, u = 2^-24: the exponential is off by 3 u at most (its instruction by 2, its argument's fraction by 1), the sum with 1, the reciprocal with its correction,
and the products by one u each (a reciprocal's error counts with the one before it): 12 u for a sigmoid times x and 16 u for gelu, whose polynomial takes nine steps; a slope is off by as much of
the sum of its terms' magnitudes.  gelu_tanh's exponent has five roundings more, 5 u of the exponent itself.
In 16 bits an approximation of 2^-15 at most is rounded once; the hardware's exponential takes what is below 2^-126 for 0, which is less than 2^-119 times x."""
import math

import pytest
import torch

import paper_2002_11082_amd as ogq
from tests import groups_reference as ref
from tests.test_groups_gpu import ACTS, DEV, ROUNDING, TYPES, near, same, say, slack_of, values

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def exact(act, x):
    """(act(x), act'(x), the sum of the magnitudes of the slope's terms, how many u they may be off by)."""
    if act == "relu":
        return x.clamp(min=0.0), (x > 0.0).double(), (x > 0.0).double(), torch.zeros_like(x)
    if act == "gelu":
        p, term = 0.5 * torch.erfc(-x / math.sqrt(2.0)), x * torch.exp(-0.5 * x * x) / math.sqrt(2.0 * math.pi)
        return x * p, p + term, p + term.abs(), torch.full_like(x, 16.0)
    w, dw = x, torch.ones_like(x)
    if act == "gelu_tanh":  # (1 + tanh(w / 2)) / 2 = 1 / (1 + exp(-w))
        c = 2.0 * math.sqrt(2.0 / math.pi)
        w, dw = c * (x + 0.044715 * x ** 3), c * (1.0 + 3.0 * 0.044715 * x * x)
    s, rest = torch.sigmoid(w), torch.sigmoid(-w)
    term = x * s * rest * dw
    return x * s, s + term, s + term.abs(), 12.0 + (8.0 * w.abs() if act == "gelu_tanh" else 0.0) + torch.zeros_like(x)


def within(out, expected, size, units, what):
    dtype = out.dtype
    if dtype == torch.float32:
        bound = units.clamp(max=2.0 ** 12) * U * size + 2.0 ** -140
    else:
        bound = 2.0 ** -15 * size + ROUNDING[dtype] * (1.0 + 2.0 ** -8) * expected.abs() + max(2.0 ** -119, torch.finfo(dtype).smallest_normal * ROUNDING[dtype])
    off = (out.double() - expected).abs() - bound
    at = off.argmax().item()
    assert bool((off <= 0.0).all()), (what, int((off > 0.0).sum()), out.flatten()[at].item(), expected.flatten()[at].item())


def all_values(dtype):
    """Every finite value of a 16-bit type; in 32 bits a dense set of those between which anything happens, and all sizes."""
    if dtype == torch.float32:
        x = torch.cat([torch.linspace(-110.0, 110.0, 1 << 20, dtype=torch.float64), torch.linspace(-15.0, 15.0, 1 << 20, dtype=torch.float64),
                       torch.logspace(-44.0, 38.4, 1 << 15, dtype=torch.float64), -torch.logspace(-44.0, 38.4, 1 << 15, dtype=torch.float64)]).float()
    else:
        x = torch.arange(-1 << 15, 1 << 15, dtype=torch.int16).view(dtype)
    x = x[torch.isfinite(x)]
    return x[: x.numel() // 256 * 256].view(-1, 256).to(DEV)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_activations_of_all_values(dtype, act):
    x = all_values(TYPES[dtype])
    say("all values", dtype, act, tuple(x.shape))
    y = ogq.ogq_activation_forward(x, ACTS[act], ogq.make_group_params(32, 8))[0]
    value, _, _, units = exact(act, x.double())
    if TYPES[dtype] == torch.float16:
        value = value.clamp(-65504.0, 65504.0)
    within(y, value, value.abs(), units, (dtype, act))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_slopes_of_all_values(dtype, act):
    """Every number of the format at every power of two between which a slope changes."""
    q = torch.arange(-127, 128, dtype=torch.float64)
    q = torch.cat([q, q[-1:]])
    x = torch.cat([q[None, :] * 2.0 ** e for e in range(-20, 2)]).view(-1, 32)
    x = x.to(TYPES[dtype]).to(DEV)
    p = ogq.make_group_params(32, 8)
    codes, exponents = ogq.ogq_group_quantize(x, p)
    held = ref.held(x, 32, 8)
    value, slope, size, units = exact(act, held)
    one = torch.ones_like(x)
    up_codes, up_exponents = ogq.ogq_group_quantize(one, p)
    within(ogq.ogq_activation_backward(one, ACTS[act], codes, exponents, p), slope, size, units, (dtype, act))
    dx, dup = ogq.ogq_activation_backward(one, ACTS[act], codes, exponents, p, up_codes, up_exponents)
    within(dx, slope, size, units, (dtype, act, "gated"))
    within(dup, value, value.abs(), units, (dtype, act, "dup"))


# A tensor larger than the chip's caches is read and written past them, by kernels of their own: as one long row, and row by row.
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_activations_larger_than_the_caches(dtype, gated):
    t = TYPES[dtype]
    for act, (rows, cols, group, pad) in zip(ACTS, ((4100, 4096, 64, 0), (2100, 8005, 128, 3), (8192, 2080, 32, 8), (4097, 4096, 128, 0))):
        say("large activation", dtype, act, gated, rows, cols, group, pad)
        p = ogq.make_group_params(group, 8)
        x, up, dy = (values(rows, cols, t, k, pad, scale=s) for k, s in ((1, 2.0), (2, 1.0), (3, 0.01)))
        if pad == 0:
            x, up, dy = x.contiguous(), up.contiguous(), dy.contiguous()
        held, u, held_up = ref.held(x, group, 8), 1.0, torch.ones(1, dtype=torch.float64, device=DEV)
        if gated:
            y, codes, exponents, up_codes, up_exponents = ogq.ogq_activation_forward(x, ACTS[act], p, up)
            dx, dup = ogq.ogq_activation_backward(dy, ACTS[act], codes, exponents, p, up_codes, up_exponents)
            u, held_up = up.double(), ref.held(up, group, 8)
            same(ogq.ogq_group_dequantize(up_codes, up_exponents, cols, p, t), held_up, "up")
        else:
            y, codes, exponents = ogq.ogq_activation_forward(x, ACTS[act], p)
            dx = ogq.ogq_activation_backward(dy, ACTS[act], codes, exponents, p)
        same(ogq.ogq_group_dequantize(codes, exponents, cols, p, t), held, "x")
        near(y, exact(act, x.double())[0] * u, slack_of(x.double(), u * x.double()), t, "y")
        value, slope = exact(act, held)[:2]
        near(dx, dy.double() * held_up * slope, slack_of(held, dy.double() * held_up), t, "dx")
        if gated:
            near(dup, dy.double() * value, slack_of(held, dy.double() * held), t, "dup")


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", TYPES)
def test_groups_larger_than_the_caches(dtype, bits):
    t = TYPES[dtype]
    for rows, cols, group, pad in ((4100, 4096, 64, 0), (2100, 8005, 128, 3), (8192, 2080, 32, 8)):
        x = values(rows, cols, t, 1, pad)
        x = x.contiguous() if pad == 0 else x
        say("large groups", dtype, bits, rows, cols, group, pad)
        p = ogq.make_group_params(group, bits)
        codes, exponents = ogq.ogq_group_quantize(x, p)
        same(ogq.ogq_group_dequantize(codes, exponents, cols, p, t), ref.held(x, group, bits), "held")
