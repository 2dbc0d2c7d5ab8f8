"""Test infrastructure: the operators of ogq_layers.h in 64 bits, written from their definitions, with bounds of how far fp32 arithmetic may be off.  Runs on the tensors' own device and shares
nothing with the kernels."""
import math

import torch

U = 2.0 ** -24  # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rounded(bound, exact, dtype):
    """`bound` before the rounding to dtype, and what that rounding adds (half a step, or half of the least subnormal)."""
    return bound + (exact.abs() + bound) * half_step(dtype) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def close(got, exact, bound, what=""):
    """`got` within `bound` (rounding included) of `exact`; NaN where exact is NaN, infinities alike."""
    got, bound = got.double(), bound.expand_as(exact)
    nan = torch.isnan(exact)
    assert torch.equal(torch.isnan(got), nan), f"{what}: NaN in other places"
    whole = torch.isinf(exact) | torch.isinf(got)
    # beyond the type's largest value: infinite on one side only where the other one is within the bound of it
    off = torch.where(nan | (got == exact), 0.0, (got - exact).abs())
    bad = ~nan & ~whole & (off > bound)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / bound.clamp(min=1e-300)).masked_fill(nan | whole, 0).max()):.3g} of the bound"
    assert torch.equal(got[whole], exact[whole]), f"{what}: infinities differ"


def norm_forward(x, weight, bias, eps):
    """y, mean, rstd, and how far y may be off before it is rounded.  With n values of a row in fp32: sums of n values have chains of at most 74 additions, so that the
    mean of the differences is off by 74 U of their mean size (at most the deviation), the variance by about 80 U of itself and the inverse root by half of that and two roundings."""
    v = x.double()
    mean = v.mean(1, keepdim=True)
    off = v - mean
    rstd = ((off * off).mean(1, keepdim=True) + eps).rsqrt()
    u = off * rstd
    w = torch.ones(x.shape[1], dtype=torch.float64, device=x.device) if weight is None else weight.double()
    y = u * w if bias is None else u * w + bias.double()
    return y, mean[:, 0], rstd[:, 0], U * ((48 * u.abs() + 80) * w.abs() + 2 * y.abs())


def norm_backward(dy, x, mean, rstd, weight):
    """dx, dweight, dbias from mean and rstd as they are given, with their bounds."""
    n, rows = x.shape[1], x.shape[0]
    r = rstd.double()[:, None]
    u = (x.double() - mean.double()[:, None]) * r
    d = dy.double()
    g = d if weight is None else d * weight.double()
    a, b = g.mean(1, keepdim=True), (g * u).mean(1, keepdim=True)
    dx = r * (g - a - u * b)
    bound = r.abs() * U * (6 * g.abs() + 80 * (g.abs().mean(1, keepdim=True) + (1 + u.abs()) * (g * u).abs().mean(1, keepdim=True)) + 6 * (u * b).abs())
    chain = (rows / 256 + 130) * U
    return (dx, bound), ((d * u).sum(0), chain * (d * u).abs().sum(0)), (d.sum(0), chain * d.abs().sum(0))


def act(name, x):
    if name is None:
        return x, torch.ones_like(x)
    if name == "relu":
        return torch.where(x > 0, x, torch.where(torch.isnan(x), x, 0.0)), torch.where(torch.isnan(x), x, (x > 0).double())
    if name == "silu":
        s = torch.sigmoid(x)
        return torch.where(x == -math.inf, 0.0, x * s), torch.where(x == math.inf, 1.0, s + x * s * torch.sigmoid(-x))
    if name == "gelu":
        p = 0.5 * torch.erfc(-x / math.sqrt(2.0))
        return x * p, p + x * torch.exp(-x * x / 2.0) / math.sqrt(2.0 * math.pi)
    u = 2.0 * math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3)
    s = torch.sigmoid(u)
    return x * s, s + x * s * torch.sigmoid(-u) * 2.0 * math.sqrt(2.0 / math.pi) * (1.0 + 3.0 * 0.044715 * x * x)


def act_bound(name, x, dtype):
    """How far act and its slope may be off for an exact x, as the header of the activations says: 16 roundings and 13 |x + 0.045 x^3| in 32 bits, 2^-15 for 16-bit types."""
    value, slope = act(name, x)
    if name is None:
        return torch.zeros_like(x), torch.zeros_like(x)
    if dtype == torch.float32:
        more = 16 + (13 * (x + 0.045 * x ** 3).abs().clamp(max=1e4) if name == "gelu_tanh" else 0)
        return U * more * value.abs() + 1e-37, U * (2 * more * slope.abs() + 8 * (1 + x.abs()) * torch.exp(-x.abs().clamp(max=40) / 2)) + 1e-37
    # (the slope's two parts may cancel, each off by 2^-15 of itself; they are at most 1.2 together, and small where |x| is large)
    return 2.0 ** -15 * value.abs() + 2.0 ** -118, 2.0 ** -15 * (slope.abs() + 1.2 * (1 + x.abs()) * torch.exp(-x.abs().clamp(max=40) / 2)) + 2.0 ** -118


def linear(x, weight, bias, activation, residual, transposed):
    """(y, bound), (before, bound): sums of K products in chains of at most K additions; fp32 products of pieces are off by 4 U (what is left out is below 2^-24 three times over)."""
    v, w = x.double(), weight.double()
    if not transposed:
        w = w.t()
    z, size = torch.mm(v, w), torch.mm(v.abs(), w.abs())
    k = x.shape[1]
    bound = U * (k + 8 + 4 * 6) * size if x.dtype == torch.float32 else U * (k + 8) * size
    if bias is not None:
        z = z + bias.double()
        bound = bound + U * 2 * (z.abs() + bias.double().abs())
    y, slope = act(activation, z)
    # the slope is at most 1.13 anywhere
    more = 1.2 * bound + act_bound(activation, z, x.dtype)[0] if activation else bound
    if residual is not None:
        y = y + residual.double()
        more = more + U * 2 * (y.abs() + residual.double().abs())
    return (y, more), (z, bound)


def embedding(tokens, table, scale):
    tokens = tokens.long()
    there = (tokens >= 0) & (tokens < table.shape[0])
    y = torch.zeros(tokens.numel(), table.shape[1], dtype=torch.float64, device=table.device)
    y[there] = table.double()[tokens[there]] * scale
    return y, 2 * U * y.abs()


def embedding_gradient(tokens, dy, vocab, scale):
    tokens = tokens.long()
    there = (tokens >= 0) & (tokens < vocab)
    one = torch.zeros(vocab, int(there.sum()), dtype=torch.float64, device=dy.device)
    one[tokens[there], torch.arange(one.shape[1], device=dy.device)] = 1.0
    d = dy.double()[there] * scale
    most = max(1, int(one.sum(1).max()) if vocab else 1)
    return one @ d, U * (min(most, 128 + most / 64) + 3) * (one @ d.abs())


def distill(logits, places, values, temperature, row_weight):
    """(loss, bound), (dlogits, bound).  With t = 1 / temperature: a logit times t is off by U of itself, its difference from the largest by U more, the exponential by 4 U (2^-17 for 16
    bits), so that q is off by (2 |z t| + |z t - most| + chain) U of itself; the same for p."""
    rows, cols = logits.shape
    z = logits.double() / temperature
    places = places.long()
    there = (places >= 0) & (places < cols)
    v = torch.where(there, values.double() / temperature, -math.inf)
    weight = torch.ones(rows, dtype=torch.float64, device=logits.device) if row_weight is None else row_weight.double()
    some = (there & (v != -math.inf)).any(1) & (weight != 0)
    at = torch.where(there, places, 0)
    log_q = z - torch.logsumexp(z, 1, keepdim=True)
    log_p = v - torch.logsumexp(v, 1, keepdim=True)
    p, q = torch.exp(log_p), torch.exp(log_q)
    p = torch.where(there, p, 0.0)
    terms = torch.where(p == 0.0, 0.0, p * (torch.where(there, log_p, 0.0) - log_q.gather(1, at)))
    loss = torch.where(some, weight * temperature ** 2 * terms.sum(1), 0.0)
    target = torch.zeros_like(z).scatter_add_(1, at, torch.where(there, p, 0.0))
    bad = torch.isnan(log_p).any(1) & there.any(1) | (v == math.inf).any(1) | torch.isnan(v).any(1) | torch.isnan(z).any(1) | (z == math.inf).any(1)
    d = torch.where(some[:, None], (q - target) * (weight * temperature)[:, None], 0.0)
    d = torch.where((some & bad)[:, None], math.nan, d)
    loss = torch.where(some & bad, math.nan, loss)
    if d.numel() == 0:
        return (loss, loss.abs()), (d, d.abs())
    finite = torch.where(torch.isinf(z), 0.0, z).abs()
    size = 3 * finite.amax(1, keepdim=True)
    exponential = 16 * U if logits.dtype == torch.float32 else 2.0 ** -17
    off_q = (2 * size + 40) * U + exponential
    vs = torch.where(torch.isfinite(v), v, 0.0).abs()
    off_p = ((6 * vs.amax(1, keepdim=True) if vs.shape[1] else 0.0) + 60 + places.shape[1]) * U
    # log q and log p are off by as much; the sum of p is 1, p is off by off_p of itself
    sizes = torch.where(p == 0.0, 0.0, p * (1 + torch.where(there & torch.isfinite(log_p), log_p, 0.0).abs() + torch.where(torch.isfinite(log_q.gather(1, at)), log_q.gather(1, at), 0.0).abs()))
    loss_bound = weight.abs() * temperature ** 2 * ((off_p * sizes.sum(1, keepdim=True))[:, 0] + (off_q + off_p)[:, 0] + 8 * U * sizes.sum(1))
    d_bound = (weight.abs() * temperature)[:, None] * ((off_q + 8 * U) * q + (off_p + 8 * U) * target)
    return (loss, torch.where(torch.isfinite(loss), loss_bound, 0.0) + U * 4 * torch.nan_to_num(loss.abs(), posinf=0.0)), (d, torch.nan_to_num(d_bound))
