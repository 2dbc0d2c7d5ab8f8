"""libogq_layers on the GPU with values from the ends of their types' ranges and far from zero, against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2002_11082_amd as ogq
from tests import layers_reference as ref
from tests.layers_layouts import LINEAR

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# a row of one piece and less, of one wavefront's registers, of a workgroup's, and longer ones
WIDTHS = [3, 8, 100, 3000, 8192, 40000]


def randn(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)


# ---------------------------------------------------------------------------------------------------------------- norm
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", WIDTHS)
def test_layer_norm_of_variances_beyond_fp32(cols, dtype):
    """rstd is 0, y the bias and dx 0 where the variance is beyond fp32; other rows are as they are alone."""
    print("[layers] norm, large variances", cols, dtype, flush=True)
    x = randn(8, cols, seed=1)
    x[1] *= 1e28
    x[2] = (x[2].sign() * 1e28)
    x[3] *= 1e36
    x[4] = 3e38
    x[4, ::4] = -3e38  # (the sum is beyond fp32, and so are differences from the mean)
    x[5] *= 3e37
    x = x.to(dtype)
    large, other = [1, 2, 3, 4, 5], [0, 6, 7]
    weight, bias, dy = 1.0 + 0.1 * randn(cols, seed=2), randn(cols, seed=3), randn(8, cols, seed=4).to(dtype)
    y, mean, rstd = ogq.ogq_layer_norm_forward(x, weight, bias)
    assert (rstd[large] == 0).all() and (y[large] == bias.to(dtype)).all()
    exact = x.double().mean(1)
    # a chain of at most 74 roundings, of sums that are at most the values' mean size
    assert bool(((mean.double() - exact).abs() <= 80 * ref.U * x.double().abs().mean(1)).all())
    want = ogq.ogq_layer_norm_forward(x[other].contiguous(), weight, bias)
    for a, b in zip((y, mean, rstd), want):
        assert torch.equal(a[other], b)
    dx, dweight, dbias = ogq.ogq_layer_norm_backward(dy, x, mean, rstd, weight)
    assert (dx[large] == 0).all()
    alone = ogq.ogq_layer_norm_backward(dy[other].contiguous(), x[other].contiguous(), want[1], want[2], weight)
    assert torch.equal(dx[other], alone[0])
    # (the large rows have no part in it; eight numbers are added in another order)
    assert bool(((dweight - alone[1]).abs() <= 8 * ref.U * (dy[other].double() * (x[other].double() - exact[other, None]) * want[2].double()[:, None]).abs().sum(0)).all())
    assert torch.isfinite(dbias).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", WIDTHS)
def test_layer_norm_of_sums_beyond_fp32(cols, dtype):
    """The variance is within fp32 and the sum of squares is not; the mean is and the sum is not."""
    x = (randn(5, cols, seed=1) * 2.0 ** 61).to(dtype)
    x[3] = 3e38
    x[4] = torch.finfo(dtype).max
    bias = randn(cols, seed=2)
    y, mean, rstd = ogq.ogq_layer_norm_forward(x, None, bias)
    exact, m, r, bound = ref.norm_forward(x[:3], None, bias, 1e-5)
    ref.close(y[:3], exact, ref.rounded(bound, exact, dtype), "y")
    ref.close(rstd[:3], r, 50 * ref.U * r, "rstd")
    ref.close(mean[:3], m, 4 * ref.U * m.abs() + 100 * ref.U / r, "mean")
    # rows of one value: the mean may be off by a few steps of it, which is what every difference is then, and nothing is left of them but the mean's second rounding
    assert torch.isfinite(mean).all() and bool(((mean[3:].double() / x[3:, 0].double()) - 1).abs().max() <= 4 * ref.U)


@pytest.mark.parametrize("cols", WIDTHS)
def test_layer_norm_of_nan(cols):
    for bad in (math.nan, math.inf, -math.inf):
        x = randn(6, cols, seed=1)
        x[2, cols // 2] = bad
        y, mean, rstd = ogq.ogq_layer_norm_forward(x)
        for t in (y, mean, rstd):
            assert torch.isfinite(t[[0, 1, 3, 4, 5]]).all()
        assert torch.isnan(y[2]).all() and torch.isnan(rstd[2]) and not torch.isfinite(mean[2])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -133])
def test_layer_norm_of_variances_below_fp32(eps, cols, dtype):
    """Values whose squares are below fp32's least number, with an eps that does not hide it."""
    x = randn(6, cols, seed=1)
    x[1] *= 2.0 ** -50
    x[2] *= 2.0 ** -60
    x[3] *= 2.0 ** -66
    x[4] *= 2.0 ** -90
    x[5] *= 2.0 ** -105
    x = x.to(dtype)
    y, mean, rstd = ogq.ogq_layer_norm_forward(x, eps=eps)
    exact, m, r, bound = ref.norm_forward(x, None, None, eps)
    ref.close(y, exact, ref.rounded(bound, exact, dtype), "y")
    ref.close(rstd, r, 50 * ref.U * r, "rstd")
    dy = randn(6, cols, seed=2).to(dtype)
    (dx, b), _, _ = ref.norm_backward(dy, x, m.float(), r.float(), None)
    ref.close(ogq.ogq_layer_norm_backward(dy, x, m.float(), r.float()), dx, ref.rounded(b, dx, dtype), "dx")


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_layer_norm_backward_far_from_zero(kind, cols):
    """Gradients are those of the exact mean, though the one that the forward pass leaves is rounded: a mean of 10^6 by up to 2^-5, a part of the deviation of 1."""
    if kind == "fp32":
        x = randn(40, cols, seed=1) + 1.0e6
    else:  # rows of 1000, in which one value is the next one
        x = torch.full((40, cols), 1000.0, device=DEV)
        x[torch.arange(40, device=DEV), torch.arange(40, device=DEV) % cols] = 1008.0
        x = x.bfloat16()
    dy = randn(40, cols, seed=2).to(x.dtype)
    _, mean, rstd = ogq.ogq_layer_norm_forward(x)
    v, d, U = x.double(), dy.double(), ref.U
    m = v.mean(1, keepdim=True)
    r = ((v - m).square().mean(1, keepdim=True) + 1e-5).rsqrt()
    u = (v - m) * r
    # u: rstd is off by 50 U, and the mean of u, whose terms are u and what the mean's rounding (half a step of it, and of its correction) makes of the deviation, has a chain of at most 74 roundings
    off_u = U * (60 * u.abs() + 100 * (u.abs().mean(1, keepdim=True) + 2 * U * m.abs() * r))
    for weight in (1.0 + 0.1 * randn(cols, seed=3), None):
        got = ogq.ogq_layer_norm_backward(dy, x, mean, rstd, weight)
        g = d if weight is None else d * weight.double()
        a, b = g.mean(1, keepdim=True), (g * u).mean(1, keepdim=True)
        dx = r * (g - a - u * b)
        off_b = (g.abs() * off_u).mean(1, keepdim=True) + 80 * U * (g * u).abs().mean(1, keepdim=True)
        bound = r * (6 * U * g.abs() + 80 * U * g.abs().mean(1, keepdim=True) + off_u * b.abs() + u.abs() * off_b) + 50 * U * dx.abs()
        ref.close(got if weight is None else got[0], dx, ref.rounded(bound, dx, x.dtype), "dx")
        if weight is not None:
            dweight = (d * u).sum(0)
            ref.close(got[1], dweight, ref.rounded((d.abs() * off_u).sum(0) + 130 * U * (d * u).abs().sum(0), dweight, torch.float32), "dweight")


# ------------------------------------------------------------------------------------------------------------- distill
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("top", [1, 20])
@pytest.mark.parametrize("rows,cols", [(300, 700), (200, 3000), (200, 30000), (60, 60000), (100, 150000)])
def test_distill_loss_far_from_zero(rows, cols, top, dtype):
    """An offset of all of a row's logits and of the teacher's values costs nothing: the loss is as exact as differences from the largest logit make it."""
    for offset, temperature in ((0.0, 1.0), (100.0, 1.5), (-1000.0, 1.0), (1000.0, 1.5), (1003.0, 1.0), (30000.0, 1.0)):
        logits = (2.0 * randn(rows, cols, seed=1) + offset).to(dtype)
        values = 2.0 * randn(rows, top, seed=2) + offset / 4
        places = torch.rand(rows, cols, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).topk(top, 1).indices
        t, U = temperature, ref.U
        z, v = logits.double() / t, values.double() / t
        z, v = z - z.amax(1, keepdim=True), v - v.amax(1, keepdim=True)
        total = z.exp().sum(1, keepdim=True)
        p = torch.softmax(v, 1)
        log_p, log_q = torch.log_softmax(v, 1), z.gather(1, places) - total.log()
        exact = t * t * (p * (log_p - log_q)).sum(1)
        # A difference is one rounding and those of the factor and of log 2, in all below 6 U of it, and its exponential is off by as much and 6 U; sums of a row's exponentials have chains of at most 60
        # additions, logarithms are off by 2 U.  The teacher's sums have as many terms as places.
        mean = ((z.exp() / total) * z.abs()).sum(1, keepdim=True)
        off_total = U * (66 + 6 * mean + 2 * total.log().abs())
        off_teacher = U * (4 + 4 * v.abs().amax(1, keepdim=True) + top)
        off = p * (6 * U * (z.gather(1, places).abs() + v.abs()) + off_total + off_teacher + 4 * U * (log_p.abs() + log_q.abs()))
        bound = t * t * (off.sum(1) + ((2 * off_teacher + min(top, 30) * U) * p * (log_p - log_q).abs()).sum(1))
        bound = bound + 4 * U * exact.abs()
        ref.close(ogq.ogq_distill_loss(logits, places, values, t), exact, bound, f"loss at {offset}")
        ref.close(ogq.ogq_distill_gradient(logits, places, values, t)[0], exact, bound, f"loss and gradient at {offset}")


# -------------------------------------------------------------------------------------------------------------- linear
# How far a slope may be off in 32 bits, in U.  silu, s (1 + x (1 - s)): 7 U and 6 U in the second term, which is at most 0.28, and two roundings.  gelu, p + x g / sqrt(2 pi): 2 U, and 5 U of at most 0.25,
# and two roundings.  gelu by tanh, s + x s (1 - s) u'(x): s is off by 7 U and by what the argument's 5 U make of it, at most 0.23 of them; the second term, at most 0.3, by 10 U and |u| (at most 4 where the term is above 0.1,
# and less than 1 / term elsewhere) times 5 U.
SLOPES = {"relu": 0, "silu": 11, "gelu": 6, "gelu_tanh": 19}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", SLOPES)
def test_bias_gradients_are_of_32_bits_in_all_types(act, dtype):
    """Of one token whose dy is 1 the bias' gradient are the slopes, in fp32 whatever the tokens' type."""
    z = torch.cat([torch.linspace(-12, 12, 20001, device=DEV), torch.linspace(3, 6, 5000, device=DEV)]).to(dtype)[None]
    dz, dbias = ogq.ogq_linear_backward(torch.ones_like(z), {"relu": ogq.RELU, "silu": ogq.SILU, "gelu": ogq.GELU, "gelu_tanh": ogq.GELU_TANH}[act], z)
    slope = ref.act(act, z[0].double())[1]
    ref.close(dbias, slope, torch.full_like(slope, SLOPES[act] * ref.U), "dbias")
    assert torch.equal(dz[0], dbias.to(dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", SLOPES)
def test_the_backward_pass_of_arguments_beyond_the_type(act, dtype):
    """An argument below fp16's values leaves -infinity for the backward pass, and an output of 0: its slope is 0; that of one above them is 1."""
    code = {"relu": ogq.RELU, "silu": ogq.SILU, "gelu": ogq.GELU, "gelu_tanh": ogq.GELU_TANH}[act]
    x, w = torch.full((5, 40), 200.0, device=DEV).to(dtype), torch.full((30, 40), 10.0, device=DEV).to(dtype)
    w[:7] = -10.0
    y, before = ogq.ogq_linear(x, w, activation=code, keep=True)
    assert (y[:, :7] == 0).all() and torch.isinf(before).all() == (dtype == torch.float16)
    dy = randn(5, 30, seed=1).to(dtype)
    dz, dbias = ogq.ogq_linear_backward(dy, code, before)
    assert (dz[:, :7] == 0).all() and torch.equal(dz[:, 7:], dy[:, 7:])
    assert (dbias[:7] == 0).all() and torch.equal(dbias, ogq.ogq_linear_backward(dz)[1])
    z = torch.where(before < 0, math.nan, before)
    dz, dbias = ogq.ogq_linear_backward(dy, code, z)
    assert torch.isnan(dz[:, :7]).all() and torch.isnan(dbias[:7]).all() and torch.equal(dz[:, 7:], dy[:, 7:])


# few tokens on the vector unit, and all that goes to the matrix cores
LAYOUTS = [(tokens, 300, 90, 0) for tokens in range(1, 9)] + [(7, 3000, 90, 0)] + LINEAR


def laid_out(values, pad):
    wide = torch.empty(values.shape[0], values.shape[1] + pad, dtype=values.dtype, device=DEV)
    wide[:, :values.shape[1]] = values
    return wide[:, :values.shape[1]]


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("tokens,outs,cols,pad", LAYOUTS)
def test_fp32_products_have_all_their_pieces(tokens, outs, cols, pad, transposed):
    """Sums of which one product is not 0.  Factors are cut into three pieces, the last below 2^-15 of the first and the second below 2^-7: the three products that are left out are below 2^-21 in all, and the sum of the six
    that are taken has at most four roundings of its size."""
    print("[layers] one product", tokens, outs, cols, pad, transposed, flush=True)
    x = torch.zeros(tokens, cols, device=DEV)
    at = torch.randint(0, cols, (tokens,), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    value, w = randn(tokens, seed=2), randn(outs, cols, seed=3)
    x[torch.arange(tokens, device=DEV), at] = value
    exact = value.double()[:, None] * w.double().t()[at]
    got = ogq.ogq_linear(laid_out(x, pad), laid_out(w.t().contiguous() if transposed else w, pad), transposed=transposed)
    ref.close(got, exact, (2.0 ** -21 + 4 * ref.U) * exact.abs(), "y")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("tokens,outs,cols,pad", LAYOUTS)
def test_linear_of_subnormal_factors(tokens, outs, cols, pad, transposed, dtype):
    """Subnormal values of x count in full: whole numbers of the type's least, times whole numbers of a large power of two, so that sums are exact.  (In fp32 of 2^-133, below which the pieces have nothing.)"""
    print("[layers] subnormal", tokens, outs, cols, pad, transposed, dtype, flush=True)
    gen = torch.Generator(device=DEV).manual_seed(1)
    least, factor = {torch.float16: (-24, 9), torch.bfloat16: (-133, 100), torch.float32: (-133, 100)}[dtype]
    a = torch.randint(-100, 101, (tokens, cols), generator=gen, device=DEV).double()
    b = torch.randint(-3, 4, (outs, cols), generator=gen, device=DEV).double()
    x, w = (a * 2.0 ** least).to(dtype), (b * 2.0 ** factor).to(dtype)
    assert bool((x != 0).eq(a != 0).all()) and float(x.double().abs().max()) < torch.finfo(dtype).smallest_normal
    weight = laid_out(w.t().contiguous() if transposed else w, pad)
    exact = torch.mm(a, b.t()) * 2.0 ** (least + factor)
    assert torch.equal(ogq.ogq_linear(laid_out(x, pad), weight, transposed=transposed), exact.to(dtype))
    # and those of the weights
    x, w = (a * 2.0 ** factor).to(dtype), (b * 2.0 ** least).to(dtype)
    weight = laid_out(w.t().contiguous() if transposed else w, pad)
    assert torch.equal(ogq.ogq_linear(laid_out(x, pad), weight, transposed=transposed), exact.to(dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("tokens,outs,cols,pad", LAYOUTS)
def test_linear_of_infinities_and_nan_in_all_layouts(tokens, outs, cols, pad, transposed, dtype):
    """They are in the sums that they belong to, in the first rows and the last, and in no others."""
    print("[layers] infinities", tokens, outs, cols, pad, transposed, dtype, flush=True)
    gen = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randint(1, 4, (tokens, cols), generator=gen, device=DEV).to(dtype)
    w = torch.randint(1, 4, (outs, cols), generator=gen, device=DEV).to(dtype)
    x[-1, 5], w[7, 5], w[-1, 5], w[9, cols - 1], x[0, cols - 1] = math.inf, -2.0, 0.0, math.nan, 2.0
    w[outs - 2, 3] = -math.inf
    exact = torch.mm(x.double(), w.double().t())
    assert torch.isnan(exact[:, 9]).all() and torch.isnan(exact[-1, -1]) and exact[-1, 7] == -math.inf and (tokens == 1 or exact[0, outs - 2] == -math.inf)
    got = ogq.ogq_linear(laid_out(x, pad), laid_out(w.t().contiguous() if transposed else w, pad), transposed=transposed)
    assert torch.equal(torch.isnan(got), torch.isnan(exact))
    assert torch.equal(got.nan_to_num(nan=0.0, posinf=math.inf, neginf=-math.inf), exact.to(dtype).nan_to_num(nan=0.0, posinf=math.inf, neginf=-math.inf))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("tokens,outs,cols,pad", LAYOUTS)
def test_linear_in_all_layouts(tokens, outs, cols, pad, transposed, dtype):
    """Sums of whole numbers are exact; with everything that happens to them on their way out, into tensors with gaps, in place of the residual."""
    print("[layers] layouts", tokens, outs, cols, pad, transposed, dtype, flush=True)
    gen = torch.Generator(device=DEV).manual_seed(3)
    x, w = (torch.randint(-3, 4, (n, cols), generator=gen, device=DEV).to(dtype) for n in (tokens, outs))
    x, w = laid_out(x, pad), laid_out(w.t().contiguous() if transposed else w, pad)
    exact = torch.mm(x.double(), w.double() if transposed else w.double().t())
    assert torch.equal(ogq.ogq_linear(x, w, transposed=transposed), exact.to(dtype))
    x = laid_out(randn(tokens, cols, seed=4).to(dtype), pad)
    w = laid_out((randn(*w.shape, seed=5) / math.sqrt(cols)).to(dtype), pad)
    bias, residual = randn(outs, seed=6), randn(tokens, outs, seed=7).to(dtype)
    for act, b, r, keep in ((None, None, None, False), ("gelu", bias, None, True), ("silu", None, residual, False), ("gelu_tanh", bias, residual, True)):
        (y, bound), (z, z_bound) = ref.linear(x, w, b, act, r, transposed)
        wide = torch.full((2, tokens, outs + 3), 55.0, dtype=dtype, device=DEV)
        out, before = wide[0, :, :outs], wide[1, :, :outs] if keep else None
        if r is not None:
            out.copy_(r)
        ogq.ogq_linear(x, w, b, None if act is None else {"gelu": ogq.GELU, "silu": ogq.SILU, "gelu_tanh": ogq.GELU_TANH}[act], None if r is None else out, transposed, y=out, before=before)
        ref.close(out, y, ref.rounded(bound, y, dtype), f"y {act}")
        if keep:
            ref.close(before, z, ref.rounded(z_bound, z, dtype), f"before {act}")
        assert (wide[:, :, outs:] == 55).all() and (keep or (wide[1] == 55).all())
        del y, bound, z, z_bound
    assert torch.equal(ogq.ogq_linear(x, w, bias, ogq.GELU_TANH, residual, transposed), out)


@pytest.mark.parametrize("cols", (1409, 1408))
def test_more_tiles_of_256_x_256_than_a_row_of_workgroups(cols):
    """More than 2^20 tiles, of rows that begin anywhere and of aligned ones: small whole numbers, so that sums are exact and each tile is a copy of the first ones."""
    torch.cuda.empty_cache()
    tokens, outs = (1 << 18) + 512, 1 << 18
    if torch.cuda.mem_get_info()[0] < 160 << 30:
        pytest.skip("less than 160 GiB of memory free")
    print("[layers] many tiles", cols, flush=True)
    gen = torch.Generator(device=DEV).manual_seed(1)
    small, w = (torch.randint(-3, 4, (512, cols), generator=gen, device=DEV).bfloat16() for _ in range(2))
    y = ogq.ogq_linear(small.repeat(tokens // 512, 1), w.repeat(outs // 512, 1))
    want = (small.double() @ w.double().T).bfloat16().repeat(1, outs // 512)
    for at in range(0, tokens, 512):
        assert torch.equal(y[at:at + 512], want), at
    del y
    torch.cuda.empty_cache()


def fastest(call, times=5):
    """us on the GPU of the fastest of several calls."""
    call()
    begin, end, least = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True), math.inf
    for _ in range(times):
        begin.record()
        call()
        end.record()
        end.synchronize()
        least = min(least, 1e3 * begin.elapsed_time(end))
    return least


@pytest.mark.parametrize("transposed", [False, True])
def test_products_of_nan_take_a_few_times_as_long(transposed):
    """A step of training that has gone wrong: NaN that come from NaN are not made again (which takes a hundred times as long)."""
    x, w = randn(2048, 2048, seed=1), randn(2048, 2048, seed=2)
    bad = torch.full_like(x, math.nan)
    assert torch.isnan(ogq.ogq_linear(bad, w, transposed=transposed)).all()
    assert fastest(lambda: ogq.ogq_linear(bad, w, transposed=transposed)) < 20 * fastest(lambda: ogq.ogq_linear(x, w, transposed=transposed))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("tokens,outs,cols", [(5, 300, 96), (70, 3000, 4096), (840, 2320, 2432), (4000, 4088, 1472), (5778, 4984, 1344)])
def test_linear_is_the_same_wherever_rows_begin(tokens, outs, cols, transposed, dtype):
    """The order of a sum is that of the sizes alone: aligned rows, which large tiles fetch another way, and rows that begin anywhere have the same sums."""
    x, w = randn(tokens, cols, seed=1).to(dtype), randn(cols if transposed else outs, outs if transposed else cols, seed=2).to(dtype)
    assert torch.equal(ogq.ogq_linear(laid_out(x, 1), laid_out(w, 3), transposed=transposed), ogq.ogq_linear(x, w, transposed=transposed))
