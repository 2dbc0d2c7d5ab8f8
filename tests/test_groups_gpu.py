"""libogq_groups on the GPU against the definitions in 64 bits (groups_reference.py).

What is held in 8 or 4 bits has to be equal.  Sums: products are exact, so the error of a sum of n terms in 32 bits is at most n * 2^-23 times
the sum of the magnitudes (every addition rounds by at most 2^-24, or by one bit more within the matrix cores), and its norm grows with the root
of n: 8 * sqrt(n) * 2^-24 times the norm of the sums of magnitudes' roots is far above it.  Both are asked for."""
import math

import pytest
import torch

import paper_2002_11082_amd as ogq
from tests import groups_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = {"relu": ogq.RELU, "gelu": ogq.GELU, "gelu_tanh": ogq.GELU_TANH, "silu": ogq.SILU}
ROUNDING = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
PIECES = {torch.float32: 3, torch.bfloat16: 1, torch.float16: 2}


def say(*what):
    print("[groups]", *what, flush=True)


def values(rows, cols, dtype, seed, pad=0, offset=0, scale=1.0):
    """Values of many sizes, rows and groups of zeros among them, as a view into a wider tensor."""
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=gen, dtype=torch.float64) * torch.exp(torch.randn(1, cols, generator=gen, dtype=torch.float64)) * scale
    if rows > 2:
        x[rows // 2] = 0.0
    x[0, : cols // 2] = 0.0
    wide = torch.full((rows, offset + cols + pad), 7.0, dtype=dtype)
    wide[:, offset:offset + cols] = x.to(dtype)
    return wide.to(DEV)[:, offset:offset + cols]


def same(a, b, what):
    assert a.shape == b.shape, what
    both_nan = torch.isnan(a.double()) & torch.isnan(b.double())
    wrong = (a.double() != b.double()) & ~both_nan
    assert not bool(wrong.any()), (what, int(wrong.sum()), wrong.nonzero()[:4].tolist())


def check_quantize(x, group, bits, what):
    say(what, tuple(x.shape), x.dtype, x.stride(), "group", group, "bits", bits)
    p = ogq.make_group_params(group, bits)
    codes, exponents = ogq.ogq_group_quantize(x, p)
    back = ogq.ogq_group_dequantize(codes, exponents, x.shape[1], p, x.dtype)
    wide = ogq.ogq_group_dequantize(codes, exponents, x.shape[1], p, torch.float32)
    numbers, expected = ref.quantize(x, group, bits)
    assert torch.equal(exponents, expected), what
    same(ref.unpack(codes, bits), numbers, what)
    assert codes.numel() == ogq.ogq_group_codes_bytes(*x.shape, p)
    held = ref.values(numbers, expected, x.shape[1])
    same(back, held, what)
    same(wide, held, what)
    return codes, exponents


SHAPES = [(1, 1), (1, 8), (3, 31), (2, 32), (5, 33), (7, 64), (4, 127), (3, 129), (1, 4096), (9, 1001), (600, 40), (2, 25088)]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", TYPES)
def test_into_groups_and_back(dtype, group, bits):
    for n, (rows, cols) in enumerate(SHAPES):
        for pad, offset in ((0, 0), (5, 0), (8, 8), (0, 3)):
            check_quantize(values(rows, cols, TYPES[dtype], 10 * n + pad, pad, offset), group, bits, f"{dtype} {pad} {offset}")


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", TYPES)
def test_every_size_of_values(dtype, bits):
    """Groups from the smallest numbers of the type to the largest, values on ties and next to the limits of an exponent."""
    t = TYPES[dtype]
    top = {"fp32": 127, "bf16": 127, "fp16": 15}[dtype]
    low = {"fp32": -149, "bf16": -133, "fp16": -24}[dtype]
    rows = []
    for e in range(low, top + 1):
        unit = 2.0 ** e
        for peak in (1.0, 1.5, 1.5 + 2.0 ** -7, 1.984375, 1.984375 + 2.0 ** -10, 1.9921875):
            row = [peak * unit * k / 32.0 * (-1) ** k for k in range(32)]
            row[0] = peak * unit
            rows.append(row)
    x = torch.tensor(rows, dtype=torch.float64).to(t)
    x = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
    largest = torch.finfo(t).max
    x = torch.cat([x, torch.full((1, 32), largest, dtype=t), torch.full((1, 32), -largest, dtype=t), torch.full((1, 32), -0.0, dtype=t)]).to(DEV)
    check_quantize(x, 32, bits, "sizes")
    halves = torch.arange(-160, 160, dtype=torch.float64) / (2.0 if bits == 8 else 20.0)  # ties of every pair of neighbours
    halves[0::32] = 127.0 if bits == 8 else 6.0
    check_quantize(halves.to(t).view(-1, 32).to(DEV), 32, bits, "ties")


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", TYPES)
def test_a_group_with_an_infinity_or_nan_stands_for_nan(dtype, bits):
    x = values(6, 200, TYPES[dtype], 3)
    x[1, 40] = math.inf
    x[2, 199] = -math.inf
    x[4, 0] = math.nan
    x[5, :] = math.nan
    codes, exponents = check_quantize(x, 64, bits, "not finite")
    assert (exponents == 255).sum().item() == 1 + 1 + 1 + 4
    back = ogq.ogq_group_dequantize(codes, exponents, 200, ogq.make_group_params(64, bits), torch.float32)
    assert torch.isnan(back[1, :64]).all() and torch.isfinite(back[1, 64:]).all()


def test_what_lies_behind_a_row_is_zero_and_the_callers_buffers_are_used():
    p = ogq.make_group_params(128, 8)
    x = values(5, 130, torch.bfloat16, 1)
    codes = torch.full((5, 256), 77, dtype=torch.uint8, device=DEV)
    exponents = torch.full((5, 2), 77, dtype=torch.uint8, device=DEV)
    a, b = ogq.ogq_group_quantize(x, p, codes, exponents)
    assert a.data_ptr() == codes.data_ptr() and b.data_ptr() == exponents.data_ptr()
    assert not codes[:, 130:].any()
    wide = torch.full((5, 200), 3.0, device=DEV)
    out = ogq.ogq_group_dequantize(codes, exponents, 130, p, torch.float32, wide[:, 7:137])
    assert out.data_ptr() == wide[:, 7:].data_ptr()
    assert (wide[:, :7] == 3.0).all() and (wide[:, 137:] == 3.0).all()
    same(wide[:, 7:137], ref.held(x, 128, 8), "view")


def test_the_same_row_again_and_again():
    """Rows of a broadcast tensor (stride 0)."""
    row = values(1, 300, torch.bfloat16, 5)
    x = row.expand(17, 300)
    check_quantize(x, 32, 8, "broadcast")
    p = ogq.make_group_params(32, 8)
    codes, exponents = ogq.ogq_group_quantize(values(17, 64, torch.bfloat16, 6), p)
    check_gradient(x, codes, exponents, 64, p, "broadcast gradient")
    row = values(1, 3905, torch.bfloat16, 7)  # (outputs that are no multiple of sixteen: nothing may be read behind the row)
    codes, exponents = ogq.ogq_group_quantize(values(700, 3300, torch.bfloat16, 8), p)
    check_gradient(row.expand(700, 3905), codes, exponents, 3300, p, "broadcast gradient")


def test_tensors_without_values():
    for rows, cols in ((0, 64), (5, 0), (0, 0)):
        p = ogq.make_group_params(32, 8)
        x = torch.empty(rows, cols, device=DEV)
        codes, exponents = ogq.ogq_group_quantize(x, p)
        assert codes.shape[0] == rows and ogq.ogq_group_dequantize(codes, exponents, cols, p, torch.float32).shape == (rows, cols)
        y, c, e, uc, ue = ogq.ogq_activation_forward(x, ogq.SILU, p, x)
        dx, dup = ogq.ogq_activation_backward(x, ogq.SILU, c, e, p, uc, ue)
        assert y.shape == dx.shape == dup.shape == (rows, cols)
    p = ogq.make_group_params(32, 8)
    codes, exponents = ogq.ogq_group_quantize(torch.empty(0, 64, device=DEV), p)
    dw = torch.full((8, 64), 5.0, device=DEV)
    assert (ogq.ogq_weight_gradient(torch.empty(0, 8, device=DEV), codes, exponents, 64, p, dw, accumulate=True) == 5.0).all()
    assert (ogq.ogq_weight_gradient(torch.empty(0, 8, device=DEV), codes, exponents, 64, p, dw) == 0.0).all()
    assert ogq.ogq_weight_gradient(torch.empty(0, 0, device=DEV), codes, exponents, 64, p).shape == (0, 64)
    p = ogq.make_group_params(32, 4)
    codes, exponents = ogq.ogq_group_quantize(torch.ones(8, 64, device=DEV), p)
    assert ogq.ogq_group_matvec(codes, exponents, 64, p, torch.empty(0, 64, device=DEV)).shape == (0, 8)
    codes, exponents = ogq.ogq_group_quantize(torch.ones(8, 0, device=DEV), p)
    assert (ogq.ogq_group_matvec(codes, exponents, 0, p, torch.empty(3, 0, device=DEV)) == torch.zeros(3, 8, device=DEV)).all()


# ----------------------------------------------------------------------------------------------------------------------
# activations
# ----------------------------------------------------------------------------------------------------------------------
def near(a, b, slack, dtype, what):
    """One rounding to the type, and `slack` for what 32 bits lose."""
    a, b = a.double(), b.double()
    tiny = torch.finfo(dtype).smallest_normal * ROUNDING[dtype] * 2.0
    off = (a - b).abs() - (ROUNDING[dtype] * b.abs() * (1.0 + 2.0 ** -8) + slack + tiny)
    assert bool((off <= 0.0).all()), (what, float(off.max()), off.argmax().item())


# A sigmoid in 32 bits is off by (|x| + 8) * 2^-24 at most times its own slope's share, the error function by 4 * 2^-24; the factors in front of
# them are at most 1 + |x|.
def slack_of(x, factor):
    return 16.0 * 2.0 ** -24 * (1.0 + x.abs()) * factor.abs()


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_activation_and_its_gradient(dtype, act, gated):
    t = TYPES[dtype]
    for n, (rows, cols, group, pad) in enumerate(((1, 1, 32, 0), (3, 100, 32, 0), (5, 257, 64, 3), (64, 256, 128, 0), (33, 520, 128, 8), (2, 4096, 64, 0))):
        say("activation", dtype, act, gated, rows, cols, group, pad)
        p = ogq.make_group_params(group, 8)
        x, up, dy = (values(rows, cols, t, 100 * n + k, pad, scale=s) for k, s in ((1, 2.0), (2, 1.0), (3, 0.01)))
        one = torch.ones(rows, cols, dtype=torch.float64, device=DEV)
        if gated:
            y, codes, exponents, up_codes, up_exponents = ogq.ogq_activation_forward(x, ACTS[act], p, up)
            dx, dup = ogq.ogq_activation_backward(dy, ACTS[act], codes, exponents, p, up_codes, up_exponents)
            u, held_up = up.double(), ref.held(up, group, 8)
            same(ogq.ogq_group_dequantize(up_codes, up_exponents, cols, p, torch.float32), held_up, "up")
        else:
            y, codes, exponents = ogq.ogq_activation_forward(x, ACTS[act], p)
            dx = ogq.ogq_activation_backward(dy, ACTS[act], codes, exponents, p)
            u, held_up = one, one
        held = ref.held(x, group, 8)
        same(ogq.ogq_group_dequantize(codes, exponents, cols, p, torch.float32), held, "x")
        near(y, ref.activation(act, x.double())[0] * u, slack_of(x.double(), u * x.double()), t, "y")
        value, slope = ref.activation(act, held)
        near(dx, dy.double() * held_up * slope, slack_of(held, dy.double() * held_up), t, "dx")
        if gated:
            near(dup, dy.double() * value, slack_of(held, dy.double() * held), t, "dup")


@pytest.mark.parametrize("act", ACTS)
def test_activation_gradient_against_differences(act):
    """(y(x + h) - y(x - h)) / 2h is off by h^2 / 6 times the third derivative (below 2 for these) and by the rounding of y."""
    h = 2.0 ** -6
    p = ogq.make_group_params(32, 8)
    x = values(4, 320, torch.float32, 9, scale=1.5)
    _, codes, exponents = ogq.ogq_activation_forward(x, ACTS[act], p)
    held = ogq.ogq_group_dequantize(codes, exponents, 320, p, torch.float32)
    dx = ogq.ogq_activation_backward(torch.ones_like(x), ACTS[act], codes, exponents, p)
    difference = (ogq.ogq_activation_forward(held + h, ACTS[act], p)[0].double() - ogq.ogq_activation_forward(held - h, ACTS[act], p)[0].double()) / (2.0 * h)
    smooth = held.abs() > h if act == "relu" else torch.ones_like(held, dtype=torch.bool)
    bound = h * h / 6.0 * 2.0 + 32.0 * 2.0 ** -24 * (1.0 + held.double().abs()) ** 2 / h
    assert ((difference - dx.double()).abs() <= bound)[smooth].all()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_activations_of_huge_and_masked_values(dtype, act):
    """Values up to the type's limits (a mask's lowest value among them): no NaN where the formula has none."""
    t = TYPES[dtype]
    big = torch.finfo(t).max
    x = torch.tensor([[big, -big, 1e4, -1e4, 100.0, -100.0, 20.0, -20.0, 0.0, -0.0] * 4], dtype=torch.float64).to(t).to(DEV).repeat(3, 1)
    p = ogq.make_group_params(32, 8)
    y, codes, exponents = ogq.ogq_activation_forward(x, ACTS[act], p)
    dx = ogq.ogq_activation_backward(torch.ones_like(x), ACTS[act], codes, exponents, p)
    assert torch.isfinite(y).all() and torch.isfinite(dx).all()
    positive = x.double() >= 20.0
    assert torch.equal(y[positive], x[positive]) and (y[x.double() <= -100.0].double().abs() < 1e-30).all()
    held = ref.held(x, 32, 8)
    assert (dx[held >= 20.0] == 1.0).all() and (dx[held <= -100.0] == 0.0).all()
    x[1, 3] = math.nan
    y, codes, exponents = ogq.ogq_activation_forward(x, ACTS[act], p)
    dx = ogq.ogq_activation_backward(torch.ones_like(x), ACTS[act], codes, exponents, p)
    assert torch.isnan(y[1, 3]) and torch.isnan(dx[1, :32]).all() and torch.isfinite(dx[1, 32:]).all() and torch.isfinite(dx[0]).all()


# ----------------------------------------------------------------------------------------------------------------------
# sums
# ----------------------------------------------------------------------------------------------------------------------
def check_sums(out, exact, magnitudes, squares, terms, what):
    """See the head of this file; out in 32 bits, magnitudes: the sums of the products' magnitudes, squares: of their squares."""
    off = (out.double() - exact).abs()
    over = off - terms * 2.0 ** -23 * magnitudes
    assert bool((over <= 0.0).all()), (what, float(over.max()), over.argmax().item())
    assert float(off.norm()) <= 8.0 * math.sqrt(terms) * 2.0 ** -24 * float(squares.sqrt().norm()) * 2.0, (what, float(off.norm()))


def check_gradient(dy, codes, exponents, cols, p, what, dw=None, accumulate=False):
    say(what, tuple(dy.shape), dy.dtype, dy.stride(), "cols", cols, "group", p.group_size, "accumulate", accumulate)
    start = dw.double() if accumulate else 0.0
    out = ogq.ogq_weight_gradient(dy, codes, exponents, cols, p, dw, accumulate)
    x = ref.values(ref.unpack(codes, 8), exponents, cols)
    d = dy.double()
    exact = d.t().contiguous() @ x + start
    magnitudes = d.abs().t().contiguous() @ x.abs() + (abs(start) if accumulate else 0.0)
    squares = (d * d).t().contiguous() @ (x * x) + (start * start if accumulate else 0.0)
    check_sums(out, exact, magnitudes, squares, PIECES[dy.dtype] * dy.shape[0] + 8, what)
    return out


GRADIENTS = [  # rows, outs, cols, group, pad
    (1, 1, 1, 32, 0), (1, 16, 32, 32, 0), (2, 7, 33, 32, 1), (31, 129, 127, 64, 0), (32, 128, 128, 128, 0), (33, 200, 333, 32, 3), (64, 64, 640, 64, 8),
    (257, 300, 130, 128, 0), (1000, 10, 1000, 32, 0), (4100, 33, 65, 64, 7), (255, 520, 264, 32, 0), (96, 1000, 40, 32, 0), (513, 256, 512, 32, 24),
    # many tiles of 256 x 256 (256 x 128 in fp32): whole steps, a part of one, one and two steps behind the loop, edges in every direction
    (640, 4096, 3136, 32, 0), (641, 4100, 3330, 64, 3), (671, 3585, 4100, 128, 0), (703, 8200, 1600, 32, 8), (1030, 3600, 4000, 32, 1), (20, 4099, 4098, 32, 0)]


# Rows shared by two teams of wavefronts: no whole step for either, one for each, an odd number, a rest of one and of two steps; parts of a sum for two teams and for one; more
# than 512 tiles, which have one team.
TEAMS = [(63, 100, 100, 32, 0), (65, 130, 260, 32, 3), (97, 20, 40, 64, 0), (129, 257, 129, 32, 0), (161, 128, 512, 128, 0), (190, 111, 222, 32, 8), (1300, 140, 150, 32, 0),
    (4097, 300, 500, 64, 1), (16390, 100, 40, 32, 0), (2300, 513, 1030, 32, 0), (70, 4001, 2700, 32, 0), (510, 3300, 2200, 128, 8)]


@pytest.mark.parametrize("rows,outs,cols,group,pad", TEAMS)
@pytest.mark.parametrize("dtype", TYPES)
def test_weight_gradient_of_teams_and_parts(dtype, rows, outs, cols, group, pad):
    test_weight_gradient(dtype, rows, outs, cols, group, pad)


@pytest.mark.parametrize("rows,outs,cols,group,pad", GRADIENTS)
@pytest.mark.parametrize("dtype", TYPES)
def test_weight_gradient(dtype, rows, outs, cols, group, pad):
    t = TYPES[dtype]
    p = ogq.make_group_params(group, 8)
    codes, exponents = ogq.ogq_group_quantize(values(rows, cols, t, 1), p)
    dy = values(rows, outs, t, 2, pad, scale=0.05)
    out = check_gradient(dy, codes, exponents, cols, p, "gradient")
    wide = torch.full((outs, cols + 5), 2.5, device=DEV)
    view = wide[:, 1:1 + cols]
    check_gradient(dy, codes, exponents, cols, p, "into a view", view)
    assert torch.equal(view, out)  # the order of a sum does not depend on where it goes
    check_gradient(dy, codes, exponents, cols, p, "added", view, True)
    assert (wide[:, 0] == 2.5).all() and (wide[:, 1 + cols:] == 2.5).all()


def test_weight_gradient_is_a_derivative():
    """The loss sum(dy * (x W^T)) is linear in W: its change along a direction is the gradient's product with it."""
    p = ogq.make_group_params(32, 8)
    x, dy = values(70, 96, torch.float32, 1), values(70, 40, torch.float32, 2)
    codes, exponents = ogq.ogq_group_quantize(x, p)
    dw = ogq.ogq_weight_gradient(dy, codes, exponents, 96, p).double()
    held = ref.held(x, 32, 8)
    gen = torch.Generator(device=DEV).manual_seed(4)
    for _ in range(5):
        w, step = (torch.randn(40, 96, generator=gen, device=DEV, dtype=torch.float64) for _ in range(2))
        loss = [(dy.double() * (held @ (w + s * step).t().contiguous())).sum() for s in (-1.0, 1.0)]
        change = float(loss[1] - loss[0]) / 2.0
        scale = float(((dy.double().abs().t().contiguous() @ held.abs()) * step.abs()).sum())
        assert abs(change - float((dw * step).sum())) <= 220 * 2.0 ** -23 * scale


@pytest.mark.parametrize("dtype", TYPES)
def test_weight_gradient_of_what_is_not_finite(dtype):
    """An infinite gradient and a group of NaN reach their own rows and columns of the result, nothing else; large finite values stay."""
    t = TYPES[dtype]
    p = ogq.make_group_params(32, 8)
    x = values(40, 96, t, 1)
    x[:, 0] = 1.0
    x[7, 40] = math.inf
    dy = values(40, 48, t, 2, scale=0.05)
    dy[3, 5] = math.inf
    dy[9, 6] = -math.inf
    dy[9, 7] = math.nan
    codes, exponents = ogq.ogq_group_quantize(x, p)
    out = ogq.ogq_weight_gradient(dy, codes, exponents, 96, p)
    assert torch.isnan(out[:, 32:64]).all()
    assert out[5, 0] == math.inf and out[6, 0] == -math.inf and torch.isnan(out[7, :]).all()
    rest = torch.ones(48, dtype=torch.bool, device=DEV)
    rest[5:8] = False
    assert torch.isfinite(out[rest][:, :32]).all() and torch.isfinite(out[rest][:, 64:]).all()
    big = torch.finfo(t).max
    dy = torch.full((2, 8), big, dtype=t, device=DEV)
    dy[1] = -big
    x = torch.tensor([[0.25] * 32, [0.125] * 32], dtype=t, device=DEV)
    codes, exponents = ogq.ogq_group_quantize(x, p)
    out = ogq.ogq_weight_gradient(dy, codes, exponents, 32, p)
    assert ((out.double() - 0.125 * big).abs() <= 2.0 ** -20 * big).all()


MATVECS = [  # tokens, outs, cols, group, pad
    (1, 1, 1, 32, 0), (1, 16, 32, 32, 0), (1, 33, 1000, 64, 0), (2, 100, 4096, 128, 0), (5, 1000, 333, 32, 1), (16, 64, 130, 64, 8), (17, 250, 520, 32, 3),
    (64, 40, 2048, 128, 0), (100, 130, 260, 64, 0), (1, 4096, 1024, 32, 0), (3, 17, 25088, 32, 0), (130, 48, 96, 32, 5), (33, 512, 4128, 32, 0),
    # many weights: stages of columns, parts of a sum, rows and columns that end inside of them
    (2, 1100, 4128, 32, 0), (16, 4100, 1025, 64, 1), (17, 2050, 2080, 32, 3), (40, 1025, 4100, 128, 0), (64, 1024, 8192, 64, 8), (150, 3000, 1440, 32, 0),
    (5, 129, 40000, 32, 2)]


@pytest.mark.parametrize("tokens,outs,cols,group,pad", MATVECS)
@pytest.mark.parametrize("dtype", TYPES)
def test_matvec(dtype, tokens, outs, cols, group, pad):
    t = TYPES[dtype]
    say("matvec", dtype, tokens, outs, cols, group, pad)
    p = ogq.make_group_params(group, 4)
    w = values(outs, cols, torch.float32, 3, scale=1.0 / math.sqrt(cols))
    codes, exponents = ogq.ogq_group_quantize(w, p)
    x = values(tokens, cols, t, 4, pad)
    held = ref.values(ref.unpack(codes, 4), exponents, cols)
    d = x.double()
    exact = d @ held.t().contiguous()
    magnitudes = d.abs() @ held.abs().t().contiguous()
    y = ogq.ogq_group_matvec(codes, exponents, cols, p, x)
    assert y.dtype == t and y.shape == (tokens, outs)
    terms = PIECES[t] * cols + 8
    if t == torch.float32:
        check_sums(y, exact, magnitudes, (d * d) @ (held * held).t().contiguous(), terms, "matvec")
    else:
        near(y, exact, terms * 2.0 ** -23 * magnitudes, t, "matvec")
    wide = torch.full((tokens, outs + 3), 2.5, dtype=t, device=DEV)
    ogq.ogq_group_matvec(codes, exponents, cols, p, x, wide[:, 1:1 + outs])
    assert torch.equal(wide[:, 1:1 + outs], y) and (wide[:, 0] == 2.5).all() and (wide[:, 1 + outs:] == 2.5).all()


# Two to four tokens, and rows so many that the wavefronts of a workgroup have different ones: one, two, three and four teams.
FEW_TOKENS = [(2, 4099, 2100, 32, 1), (3, 8190, 500, 64, 0), (4, 6145, 999, 128, 8), (1, 8193, 2080, 32, 0), (1, 4097, 33, 32, 2), (2, 37, 6200, 64, 0),
    (4, 1, 1, 32, 0), (3, 2050, 8160, 32, 0), (2, 8200, 1000, 32, 0)]


@pytest.mark.parametrize("tokens,outs,cols,group,pad", FEW_TOKENS)
@pytest.mark.parametrize("dtype", TYPES)
def test_matvec_of_few_tokens(dtype, tokens, outs, cols, group, pad):
    test_matvec(dtype, tokens, outs, cols, group, pad)


@pytest.mark.parametrize("tokens", [1, 2, 5, 40])
@pytest.mark.parametrize("dtype", TYPES)
def test_products_of_the_smallest_values(dtype, tokens):
    """Subnormal values: each may lose what it has below 2^-133 (times a weight of at most 6 * 2^e), and a sum its last bit."""
    t = TYPES[dtype]
    p = ogq.make_group_params(32, 4)
    codes, exponents = ogq.ogq_group_quantize(values(50, 300, torch.float32, 3), p)
    held = ref.values(ref.unpack(codes, 4), exponents, 300)
    x = (values(tokens, 300, torch.float32, 5) * 2.0 ** (-130 if t != torch.float16 else -20)).to(t)
    exact = x.double() @ held.t().contiguous()
    y = ogq.ogq_group_matvec(codes, exponents, 300, p, x).double()
    terms, last = (x.double().abs() @ held.abs().t().contiguous()) * 300 * 2.0 ** -23, 2.0 ** (-149 if t == torch.float32 else -133 if t == torch.bfloat16 else -24)
    assert ((y - exact).abs() <= terms + 300 * (2.0 ** -133 * held.abs().max() + 2.0 ** -149) + exact.abs() * 2.0 ** -8 + last).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_matvec_of_what_is_not_finite(dtype):
    t = TYPES[dtype]
    p = ogq.make_group_params(32, 4)
    w = values(40, 96, torch.float32, 3, scale=0.1)
    w[:, 0] = 1.0
    w[11, 50] = math.nan
    codes, exponents = ogq.ogq_group_quantize(w, p)
    x = values(4, 96, t, 4)
    x[1, 0] = math.inf
    x[2, 3] = math.nan
    y = ogq.ogq_group_matvec(codes, exponents, 96, p, x)
    assert torch.isnan(y[:, 11]).all() and torch.isnan(y[2]).all()
    keep = torch.arange(40, device=DEV) != 11
    assert torch.isfinite(y[0, keep]).all() and torch.isfinite(y[3, keep]).all()
    assert (y[1, keep] == math.inf).all()


# ----------------------------------------------------------------------------------------------------------------------
# long tensors, streams, graphs
# ----------------------------------------------------------------------------------------------------------------------
def test_offsets_beyond_32_bits():
    """Tensors of more than 2^32 values: the last rows against the same rows alone."""
    rows, cols = (1 << 17) + 3, 1 << 15
    say("long", rows, cols)
    p = ogq.make_group_params(32, 8)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    x[:5].normal_()
    x[-5:].normal_()
    x[5:-5] = 1.0
    for pad in (0, 1):  # as one long row, and row by row
        v = x if pad == 0 else x[:, :cols - 1]
        codes, exponents = ogq.ogq_group_quantize(v, p)
        for part in (slice(0, 5), slice(rows - 5, rows)):
            c, e = ogq.ogq_group_quantize(v[part].contiguous(), p)
            assert torch.equal(codes[part], c) and torch.equal(exponents[part], e)
        back = ogq.ogq_group_dequantize(codes, exponents, v.shape[1], p, torch.bfloat16)
        same(back[-5:], ref.held(v[-5:], 32, 8), "back")
        assert (back[1000:1010] == 1.0).all()
        del back
    # 4-bit weights with as many values: the last outputs
    p4 = ogq.make_group_params(32, 4)
    codes, exponents = ogq.ogq_group_quantize(x, p4)
    t = values(2, cols, torch.float32, 8)
    y = ogq.ogq_group_matvec(codes, exponents, cols, p4, t)
    c, e = codes[-5:].contiguous(), exponents[-5:].contiguous()
    held = ref.values(ref.unpack(c, 4), e, cols)
    off = (y[:, -5:].double() - t.double() @ held.t().contiguous()).abs()
    assert (off <= (3 * cols + 8) * 2.0 ** -23 * (t.double().abs() @ held.abs().t().contiguous())).all()


def test_weight_gradient_of_a_long_sum():
    """More than 2^32 values of dy; all but a few rows are 0."""
    rows, outs, cols = (1 << 21) + 5, 2048, 64
    say("long sum", rows)
    p = ogq.make_group_params(64, 8)
    dy = torch.zeros(rows, outs, dtype=torch.bfloat16, device=DEV)
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    at = torch.tensor([0, 1, rows // 2, rows - 2, rows - 1], device=DEV)
    dy[at] = values(5, outs, torch.bfloat16, 1)
    x[at] = values(5, cols, torch.bfloat16, 2)
    codes, exponents = ogq.ogq_group_quantize(x, p)
    out = ogq.ogq_weight_gradient(dy, codes, exponents, cols, p)
    exact = dy[at].double().t().contiguous() @ ref.held(x[at], 64, 8)
    assert ((out.double() - exact).abs() <= 16 * 2.0 ** -23 * (dy[at].double().abs().t().contiguous() @ ref.held(x[at], 64, 8).abs())).all()


def _step(x, up, dy, w_codes, w_exponents, p, p4):
    y, codes, exponents, up_codes, up_exponents = ogq.ogq_activation_forward(x, ogq.SILU, p, up)
    dx, dup = ogq.ogq_activation_backward(dy, ogq.SILU, codes, exponents, p, up_codes, up_exponents)
    dw = ogq.ogq_weight_gradient(dx, codes, exponents, x.shape[1], p)
    z = ogq.ogq_group_matvec(w_codes, w_exponents, x.shape[1], p4, y[:5])
    return y, dx, dup, dw, z


def _inputs(seed):
    x, up, dy = (values(600, 256, torch.bfloat16, seed + k) for k in range(3))
    w_codes, w_exponents = ogq.ogq_group_quantize(values(300, 256, torch.float32, seed + 3), ogq.make_group_params(32, 4))
    return x.contiguous(), up.contiguous(), dy.contiguous(), w_codes, w_exponents


def test_results_repeat_on_another_stream():
    p, p4 = ogq.make_group_params(64, 8), ogq.make_group_params(32, 4)
    inputs = _inputs(1)
    first = _step(*inputs, p, p4)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        for _ in range(5):
            again = _step(*inputs, p, p4)
    stream.synchronize()
    for a, b in zip(first, again):
        assert torch.equal(a, b)


def test_captured_in_a_graph():
    p, p4 = ogq.make_group_params(64, 8), ogq.make_group_params(32, 4)
    kept = _inputs(1)
    _step(*kept, p, p4)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _step(*kept, p, p4)
    for seed in (20, 30, 40):
        new = _inputs(seed)
        for a, b in zip(kept, new):
            a.copy_(b)
        graph.replay()
        eager = _step(*new, p, p4)
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b)


def test_the_example_learns_and_serves():
    from paper_2002_11082_amd import checkpointed_block
    losses, block = checkpointed_block.train(128, 256, 128, 2, 40, tell=lambda text: say(text))
    assert losses[-1] < 0.2 * losses[0], (losses[0], losses[-1])
    x = torch.randn(5, 128, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).bfloat16()
    exact = block.plain(x)
    assert float((checkpointed_block.Served(block)(x).float() - exact).norm()) < 0.4 * float(exact.norm())
