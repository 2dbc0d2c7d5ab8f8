"""Test infrastructure: the format and the operators of ogq_groups.h in 64 bits, written from their definitions.  Runs on the
tensors' own device and shares nothing with the kernels."""
import math

import torch

LARGEST = {8: 127.0, 4: 6.0}
NUMBERS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
LIMITS = {(8, torch.float16): (-24, 9), (4, torch.float16): (-23, 13)}


def limits(bits, dtype):
    return LIMITS.get((bits, dtype), (-126, 121) if bits == 8 else (-125, 125))


def power(e):
    """2^e in 64 bits, from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _grouped(x, group):
    rows, cols = x.shape
    groups = -(-cols // group)
    v = torch.zeros(rows, groups * group, dtype=torch.float64, device=x.device)
    v[:, :cols] = x.double()
    return v.view(rows, groups, group)


def quantize(x, group, bits):
    """(codes as the numbers in units of the shared power [rows, groups * group], exponent bytes [rows, groups])."""
    rows = x.shape[0]
    v = _grouped(x, group)
    most = v.abs().amax(2)
    finite = torch.isfinite(v).all(2)
    most = torch.where(finite, most, torch.ones_like(most))
    low, high = limits(bits, x.dtype)
    # the smallest e with most <= Q * 2^e, found by trying: from the logarithm's neighbourhood upwards
    e = torch.floor(torch.log2(torch.clamp(most, min=1e-300) / LARGEST[bits])).long() - 1
    e = e.clamp(-1000, 1000)
    for _ in range(3):
        e = torch.where(most > LARGEST[bits] * power(e), e + 1, e)
    e = torch.where(most == 0.0, torch.full_like(e, low), e).clamp(low, high)
    t = (v / power(e)[..., None]).clamp(-LARGEST[bits], LARGEST[bits])
    t = torch.where(finite[..., None], t, torch.zeros_like(t))
    if bits == 8:
        q = torch.round(t)  # ties to even
    else:
        grid = torch.tensor(NUMBERS, dtype=torch.float64, device=x.device)
        distance = (t.abs()[..., None] - grid).abs()
        nearest = distance.amin(-1, keepdim=True)
        index = torch.arange(8, device=x.device)
        # of two numbers at the same distance the one with the even index
        index = torch.where(distance == nearest, index + 100 * (index % 2), 1000).argmin(-1)
        q = grid[index] * torch.where(t < 0.0, -1.0, 1.0)
    byte = torch.where(finite, e + 127, 255)
    return q.view(rows, -1), byte.to(torch.uint8)


def unpack(codes, bits):
    """The numbers that stored codes are, in units of the shared power."""
    if bits == 8:
        return codes.view(torch.int8).double()
    table = torch.tensor(NUMBERS, dtype=torch.float64, device=codes.device)
    table = torch.cat([table, -table])
    both = torch.stack([codes & 15, codes >> 4], 2).view(codes.shape[0], -1)
    return table[both.long()]


def values(numbers, exponents, cols):
    """What numbers and exponent bytes stand for, [rows, cols]."""
    rows, groups = exponents.shape
    unit = power(exponents.long() - 127)
    unit = torch.where(exponents == 255, torch.full_like(unit, math.nan), unit)
    return (numbers.view(rows, groups, -1) * unit[..., None]).view(rows, -1)[:, :cols]


def held(x, group, bits):
    return values(*quantize(x, group, bits), x.shape[1])


def activation(name, x):
    """(act(x), act'(x)) in 64 bits."""
    if name == "relu":
        return torch.where(x < 0.0, torch.zeros_like(x), x), torch.where(x > 0.0, torch.ones_like(x), torch.zeros_like(x))
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-x))
        return x * s, s + x * s * (1.0 - s)
    if name == "gelu":
        p = 0.5 * torch.erfc(-x / math.sqrt(2.0))
        return x * p, p + x * torch.exp(-0.5 * x * x) / math.sqrt(2.0 * math.pi)
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (x + 0.044715 * x ** 3))
    return 0.5 * x * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * x * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * x * x)
