"""Sums of libogq_groups (weight gradients, products with 4-bit weights) where layouts, values and types are at their limits, on the GPU against the
definitions in 64 bits.  Bounds as in test_groups_gpu.py: n terms summed in 32 bits are off by at most n * 2^-23 times the sum of their magnitudes."""
import math

import pytest
import torch

import paper_2002_11082_amd as ogq
from tests import groups_reference as ref
from tests.test_groups_gpu import DEV, PIECES, ROUNDING, TYPES, check_gradient, say, values

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------------------------------------------------------------
# the smallest values
# ----------------------------------------------------------------------------------------------------------------------
def flushed(x):
    """x without the values that a unit without subnormal numbers takes for 0."""
    return torch.where(x.abs() < torch.finfo(x.dtype).smallest_normal, torch.zeros_like(x), x)


def lost(x):
    """What a value in 32 bits may lose in three pieces of bf16, of which 2^-133 is the smallest."""
    return torch.clamp(x.abs(), max=2.0 ** -133) if x.dtype == torch.float32 else torch.zeros_like(x)


# The values' scale: subnormal numbers for the most part, and (in 32 bits) numbers whose second and third pieces are.
TINY = {torch.float32: (2.0 ** -128, 2.0 ** -120), torch.bfloat16: (2.0 ** -128,), torch.float16: (2.0 ** -17,)}


def bounded(out, x, w, scale, what):
    """out against x @ w^T of positive values, by a bound that would see that small values are lost."""
    d = x.double()
    exact = d @ w.t().contiguous()
    dtype = out.dtype
    bound = (PIECES[x.dtype] * x.shape[1] + 8) * (2.0 ** -23 * exact + 2.0 ** -149) + lost(x).double() @ w.t().contiguous()
    if dtype != torch.float32:
        bound = bound * (1.0 + ROUNDING[dtype]) + ROUNDING[dtype] * exact + torch.finfo(dtype).smallest_normal * ROUNDING[dtype]
    assert bool((exact > 2.0 * bound).all()), what  # zeros would be seen
    if scale < torch.finfo(x.dtype).smallest_normal:
        assert bool((exact - flushed(x).double() @ w.t().contiguous() > bound).all()), what
    off = (out.double() - exact).abs() - bound
    assert bool((off <= 0.0).all()), (what, float((off / exact).max()), int((off > 0.0).sum()))


def positive(rows, cols, dtype, seed, scale):
    gen = torch.Generator().manual_seed(seed)
    return ((0.25 + torch.rand(rows, cols, generator=gen, dtype=torch.float64)) * scale).to(dtype).to(DEV)


@pytest.mark.parametrize("tokens,outs,cols", [(1, 50, 300), (2, 50, 300), (4, 50, 300), (5, 50, 300), (40, 50, 300), (40, 1024, 4096), (100, 130, 520)])
@pytest.mark.parametrize("dtype", TYPES)
def test_products_keep_subnormal_values(dtype, tokens, outs, cols):
    t = TYPES[dtype]
    p = ogq.make_group_params(32, 4)
    codes, exponents = ogq.ogq_group_quantize(positive(outs, cols, torch.float32, 3, 1.0), p)
    held = ref.values(ref.unpack(codes, 4), exponents, cols)
    for scale in TINY[t]:
        say("subnormal tokens", dtype, tokens, outs, cols, scale)
        x = positive(tokens, cols, t, 4, scale)
        bounded(ogq.ogq_group_matvec(codes, exponents, cols, p, x), x, held, scale, (dtype, tokens, scale))


@pytest.mark.parametrize("rows,outs,cols", [(1, 16, 32), (50, 40, 100), (200, 300, 333), (4100, 33, 65), (640, 4096, 2560)])
@pytest.mark.parametrize("dtype", TYPES)
def test_weight_gradients_keep_subnormal_values(dtype, rows, outs, cols):
    t = TYPES[dtype]
    p = ogq.make_group_params(32, 8)
    codes, exponents = ogq.ogq_group_quantize(positive(rows, cols, t, 3, 1.0), p)
    held = ref.values(ref.unpack(codes, 8), exponents, cols)
    for scale in TINY[t]:
        say("subnormal gradients", dtype, rows, outs, cols, scale)
        dy = positive(rows, outs, t, 4, scale)
        out = ogq.ogq_weight_gradient(dy, codes, exponents, cols, p)
        bounded(out, dy.t(), held.t().contiguous(), scale, (dtype, rows, scale))


@pytest.mark.parametrize("dtype", TYPES)
def test_factors_held_next_to_the_least_exponent(dtype):
    """Checkpoints and weights whose shared power is the smallest that there is, next to it, or above it by little."""
    t = TYPES[dtype]
    for low in ((2.0 ** -20, 2.0 ** -16) if t == torch.float16 else (2.0 ** -122, 2.0 ** -118)):
        p = ogq.make_group_params(32, 8)
        codes, exponents = ogq.ogq_group_quantize(positive(70, 100, t, 3, low), p)
        held = ref.values(ref.unpack(codes, 8), exponents, 100)
        dy = positive(70, 60, t, 4, 64.0)
        bounded(ogq.ogq_weight_gradient(dy, codes, exponents, 100, p), dy.t(), held.t().contiguous(), 1.0, (dtype, low))
    p = ogq.make_group_params(32, 4)
    codes, exponents = ogq.ogq_group_quantize(positive(60, 100, torch.float32, 3, 2.0 ** -123), p)
    held = ref.values(ref.unpack(codes, 4), exponents, 100)
    for tokens in (1, 3, 20):
        x = positive(tokens, 100, t, 4, 64.0)
        if t == torch.float16:  # (the sums are below the least fp16: they round to 0)
            assert not ogq.ogq_group_matvec(codes, exponents, 100, p, x).any()
        else:
            bounded(ogq.ogq_group_matvec(codes, exponents, 100, p, x), x, held, 1.0, (dtype, tokens))


# ----------------------------------------------------------------------------------------------------------------------
# the order of a sum
# ----------------------------------------------------------------------------------------------------------------------
def layouts(x):
    """The same values with rows next to each other, apart by little, and far apart."""
    rows, cols = x.shape
    yield "contiguous", x
    for stride in (cols + 1, cols + 8, 64 + cols, 1 << 24):
        if rows * stride < 1 << 31:
            wide = torch.empty((rows - 1) * stride + cols, dtype=x.dtype, device=DEV).as_strided((rows, cols), (stride, 1))
            wide.copy_(x)
            yield f"stride {stride}", wide


@pytest.mark.parametrize("rows,outs,cols", [(200, 10, 1000), (97, 10, 33), (129, 130, 260), (190, 7, 222), (255, 128, 128), (1300, 13, 150), (2300, 12, 1030), (700, 3, 4000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_the_order_of_a_gradients_sum_does_not_depend_on_strides(dtype, rows, outs, cols):
    p = ogq.make_group_params(32, 8)
    codes, exponents = ogq.ogq_group_quantize(values(rows, cols, TYPES[dtype], 1), p)
    dy = values(rows, outs, TYPES[dtype], 2, scale=0.05).contiguous()
    first = check_gradient(dy, codes, exponents, cols, p, "order")
    for name, view in layouts(dy):
        say("order", dtype, rows, outs, cols, name)
        assert torch.equal(ogq.ogq_weight_gradient(view, codes, exponents, cols, p), first), name
    one = dy[rows // 3:rows // 3 + 1].expand(rows, outs)
    assert torch.equal(ogq.ogq_weight_gradient(one, codes, exponents, cols, p), ogq.ogq_weight_gradient(one.contiguous(), codes, exponents, cols, p))


# ----------------------------------------------------------------------------------------------------------------------
# fp16 gradients
# ----------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,outs,cols", [(1, 16, 32), (40, 48, 96), (33, 200, 333), (200, 10, 1000), (129, 257, 129), (4100, 33, 65), (1300, 140, 150), (641, 4100, 2570)])
@pytest.mark.parametrize("held_as", ["bf16", "fp32"])
def test_fp16_gradients_with_a_checkpoint_of_another_type(held_as, rows, outs, cols):
    """Inputs beyond what fp16 holds, at both ends, beside ordinary ones."""
    p = ogq.make_group_params(32, 8)
    x = values(rows, cols, torch.float32, 1)
    powers = torch.tensor([2.0 ** 20, 1.0, 2.0 ** -30, 2.0 ** 8, 2.0 ** 60, 2.0 ** -100])
    for n, column in enumerate(range(0, cols, 32)):
        x[:, column:column + 32] *= float(powers[n % 6])
    x[rows // 2, :32] = 3.0 * 2.0 ** 12  # (one group of a column alone)
    codes, exponents = ogq.ogq_group_quantize(x.to(TYPES[held_as]), p)
    dy = values(rows, outs, torch.float16, 2, scale=0.05)
    check_gradient(dy, codes, exponents, cols, p, "other type")
    x = values(rows, cols, torch.float32, 1) * 0.01
    x[-1, -1] = 1e6  # one value in the whole checkpoint
    codes, exponents = ogq.ogq_group_quantize(x.to(TYPES[held_as]), p)
    check_gradient(dy, codes, exponents, cols, p, "one group")


# ----------------------------------------------------------------------------------------------------------------------
# what the matrix cores and cut sums make of infinities and NaN; gradients added past the caches
# ----------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("tokens,outs,cols", [(1, 40, 96), (2, 40, 96), (4, 40, 96), (5, 40, 96), (17, 40, 96), (40, 40, 96), (100, 40, 96), (40, 1024, 4128), (7, 129, 40000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_products_of_what_is_not_finite(dtype, tokens, outs, cols):
    t = TYPES[dtype]
    say("not finite", dtype, tokens, outs, cols)
    p = ogq.make_group_params(32, 4)
    w = values(outs, cols, torch.float32, 3, scale=0.1)
    w[:, 0] = 1.0
    w[:, 1:32] = w[:, 1:32].clamp(-4.0, 4.0)  # (so that the first column's 1 is not lost in its group)
    w[11, 50] = math.nan
    codes, exponents = ogq.ogq_group_quantize(w, p)
    x = values(tokens, cols, t, 4)
    at_inf, at_nan, at_low = tokens - 1, tokens // 2, tokens // 3
    x[at_inf, 0] = math.inf
    if tokens > 2:
        x[at_nan, cols - 1] = math.nan
        x[at_low, 0] = -math.inf
    y = ogq.ogq_group_matvec(codes, exponents, cols, p, x)
    keep = torch.arange(outs, device=DEV) != 11
    assert torch.isnan(y[:, 11]).all()
    assert (y[at_inf, keep] == math.inf).all()
    rest = torch.ones(tokens, dtype=torch.bool, device=DEV)
    rest[at_inf] = False
    if tokens > 2:
        assert torch.isnan(y[at_nan]).all()
        rest[at_nan] = rest[at_low] = False
        if at_low != at_nan:
            assert (y[at_low, keep] == -math.inf).all()
    assert torch.isfinite(y[rest][:, keep]).all()


@pytest.mark.parametrize("rows,outs,cols", [(40, 2050, 4096), (33, 2048, 4112), (700, 4096, 4096)])
@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_added_to_large_sums(dtype, rows, outs, cols):
    """More sums than the caches hold, in rows of whole lines: into new ones, and added to what is there."""
    p = ogq.make_group_params(64, 8)
    codes, exponents = ogq.ogq_group_quantize(values(rows, cols, TYPES[dtype], 1), p)
    dy = values(rows, outs, TYPES[dtype], 2, scale=0.05)
    dw = torch.full((outs, cols), 2.5, device=DEV)
    first = check_gradient(dy, codes, exponents, cols, p, "large", dw).clone()
    check_gradient(dy, codes, exponents, cols, p, "large, added", dw, True)
    assert torch.equal(dw, first + first)
