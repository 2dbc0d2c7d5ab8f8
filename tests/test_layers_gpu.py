"""libogq_layers on the GPU, against its formulas in 64 bits: odd sizes, strides, views, empty tensors, infinities and NaN, gradients, streams and captured graphs."""
import math

import pytest
import torch

import paper_2002_11082_amd as ogq
from tests import layers_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
ACTS = {None: None, "relu": ogq.RELU, "gelu": ogq.GELU, "gelu_tanh": ogq.GELU_TANH, "silu": ogq.SILU}


def values(rows, cols, dtype, seed, pad=0, shift=0, factor=1.0, offset=0.0):
    """Random values as rows of a wider tensor, `shift` values behind its start."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    wide = torch.full((rows, cols + pad + shift), 77.0, dtype=dtype, device=DEV)
    x = wide[:, shift:shift + cols]
    x.copy_(torch.randn(rows, cols, generator=gen, device=DEV) * factor + offset)
    return x


def vector(n, seed, factor=1.0, offset=0.0):
    return torch.randn(n, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV) * factor + offset


def whole(rows, cols, dtype, seed, most=3):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-most, most + 1, (rows, cols), generator=gen, device=DEV).to(dtype)


# ---------------------------------------------------------------------------------------------------------------- norm
NORMS = [(1, 1, 0), (3, 2, 1), (5, 7, 0), (2, 8, 0), (9, 33, 3), (4, 64, 0), (7, 500, 5), (6, 512, 0), (5, 513, 0), (3, 1001, 7), (4, 1024, 0), (3, 2047, 1), (3, 2049, 0), (2, 4096, 0),
         (3, 5000, 8), (2, 8192, 0), (2, 8193, 3), (2, 16384, 0), (2, 16387, 1), (2, 32768, 0), (2, 32769, 0), (1, 70001, 0), (300, 96, 0), (1237, 200, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad", NORMS)
def test_layer_norm(rows, cols, pad, dtype):
    print("[layers] norm", rows, cols, pad, dtype, flush=True)
    x = values(rows, cols, dtype, 1, pad, shift=pad % 3, offset=0.5)
    for weight, bias in ((None, None), (vector(cols, 2, 0.3, 1.0), vector(cols, 3)), (vector(cols, 4), None)):
        y, mean, rstd = ogq.ogq_layer_norm_forward(x, weight, bias, 1e-5)
        exact, m, r, bound = ref.norm_forward(x, weight, bias, 1e-5)
        ref.close(y, exact, ref.rounded(bound, exact, dtype), "y")
        ref.close(mean, m, 4 * ref.U * m.abs() + 100 * ref.U / r, "mean")
        ref.close(rstd, r, 50 * ref.U * r, "rstd")
        dy = values(rows, cols, dtype, 5, pad)
        mean, rstd = m.float(), r.float()
        out = ogq.ogq_layer_norm_backward(dy, x, mean, rstd, weight)
        (dx, b), (dw, bw), (db, bb) = ref.norm_backward(dy, x, mean, rstd, weight)
        ref.close(out if weight is None else out[0], dx, ref.rounded(b, dx, dtype), "dx")
        if weight is not None:
            ref.close(out[1], dw, ref.rounded(bw, dw, torch.float32), "dweight")
            ref.close(out[2], db, ref.rounded(bb, db, torch.float32), "dbias")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(5000, 40), (2100, 300), (700, 4096), (1100, 16384), (40, 33000)])
def test_sums_of_layer_norm_over_many_rows(rows, cols, dtype):
    print("[layers] norm, many rows", rows, cols, dtype, flush=True)
    x, dy, weight = values(rows, cols, dtype, 1), values(rows, cols, dtype, 2), vector(cols, 3)
    _, m, r, _ = ref.norm_forward(x, weight, None, 1e-5)
    mean, rstd = m.float(), r.float()
    dx, dweight, dbias = ogq.ogq_layer_norm_backward(dy, x, mean, rstd, weight)
    (ex, b), (ew, bw), (eb, bb) = ref.norm_backward(dy, x, mean, rstd, weight)
    ref.close(dx, ex, ref.rounded(b, ex, dtype), "dx")
    ref.close(dweight, ew, ref.rounded(bw, ew, torch.float32), "dweight")
    ref.close(dbias, eb, ref.rounded(bb, eb, torch.float32), "dbias")
    # added to what is there, and the same from call to call
    again = [torch.full_like(dweight, 2.0), torch.full_like(dbias, -3.0)]
    ogq.ogq_layer_norm_backward(dy, x, mean, rstd, weight, dweight=again[0], dbias=again[1], accumulate=True)
    assert torch.equal(again[0], dweight + 2.0) and torch.equal(again[1], dbias - 3.0)
    # in place of dy
    place = dy.clone()
    assert ogq.ogq_layer_norm_backward(place, x, mean, rstd, weight, dx=place)[0] is not None
    assert torch.equal(place, dx)


def test_layer_norm_of_far_offsets_and_bad_rows():
    x = values(6, 1000, torch.float32, 1, offset=1.0e6)
    y, mean, rstd = ogq.ogq_layer_norm_forward(x)
    exact, m, r, bound = ref.norm_forward(x, None, None, 1e-5)
    ref.close(y, exact, ref.rounded(bound, exact, torch.float32), "y")
    x = values(6, 1000, torch.bfloat16, 2)
    x[1, 3], x[2, 5], x[3] = math.nan, math.inf, 4.0
    y, mean, rstd = ogq.ogq_layer_norm_forward(x, None, vector(1000, 3))
    assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all() and torch.equal(y[3], vector(1000, 3).bfloat16())
    assert torch.isfinite(y[[0, 4, 5]].float()).all()


def test_layer_norm_over_nothing():
    dw, db = torch.full((5,), 9.0, device=DEV), torch.full((5,), 9.0, device=DEV)
    none = torch.empty(0, device=DEV)
    x = torch.empty(0, 5, device=DEV)
    assert ogq.ogq_layer_norm_forward(x)[0].shape == (0, 5)
    ogq.ogq_layer_norm_backward(x, x, none, none, vector(5, 1), dweight=dw, dbias=db, accumulate=True)
    assert (dw == 9).all() and (db == 9).all()
    ogq.ogq_layer_norm_backward(x, x, none, none, vector(5, 1), dweight=dw, dbias=db)
    assert (dw == 0).all() and (db == 0).all()
    x = torch.empty(4, 0, device=DEV)
    assert ogq.ogq_layer_norm_forward(x)[0].shape == (4, 0)


# -------------------------------------------------------------------------------------------------------------- linear
LINEARS = [(1, 1, 1), (1, 5, 3), (2, 8, 16), (3, 100, 33), (4, 300, 600), (5, 17, 1000), (6, 2100, 130), (7, 64, 2050), (8, 513, 777), (1, 9000, 40), (9, 1, 1), (9, 130, 65), (16, 128, 64),
           (33, 200, 31), (64, 129, 127), (65, 128, 128), (100, 300, 257), (129, 127, 320), (200, 1000, 96), (300, 40, 3000), (12, 16, 5000)]
# few tokens: a wavefront's four rows of weights, a workgroup's, and what goes to the matrix cores
LINEARS += [(tokens, 8197, 70) for tokens in range(1, 9)] + [(tokens, 2051, 300) for tokens in range(1, 9)] + [(tokens, 8197, 2056) for tokens in (1, 4, 5)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("tokens,outs,cols", LINEARS)
def test_linear(tokens, outs, cols, transposed, dtype):
    print("[layers] linear", tokens, outs, cols, transposed, dtype, flush=True)
    pad = (tokens + outs + cols) % 5
    x = values(tokens, cols, dtype, 1, pad, shift=pad % 2)
    w = values(cols if transposed else outs, outs if transposed else cols, dtype, 2, (pad * 3) % 4, shift=pad % 3, factor=1.0 / math.sqrt(cols))
    bias, residual = vector(outs, 3), values(tokens, outs, dtype, 4, pad)
    for act, b, r in ((None, None, None), ("gelu", bias, None), ("silu", None, residual), ("relu", bias, residual), ("gelu_tanh", bias, residual)):
        (y, bound), (z, z_bound) = ref.linear(x, w, b, act, r, transposed)
        got, before = ogq.ogq_linear(x, w, b, ACTS[act], r, transposed, keep=True)
        ref.close(got, y, ref.rounded(bound, y, dtype), f"y {act}")
        ref.close(before, z, ref.rounded(z_bound, z, dtype), f"before {act}")
        assert torch.equal(ogq.ogq_linear(x, w, b, ACTS[act], r, transposed), got)
    # outputs of the caller, in wider tensors whose other values stay
    wide = torch.full((tokens, outs + 5), 55.0, dtype=dtype, device=DEV)
    out = wide[:, 2:2 + outs]
    ogq.ogq_linear(x, w, bias, None, residual, transposed, y=out)
    assert torch.equal(out, ogq.ogq_linear(x, w, bias, None, residual, transposed))
    assert (wide[:, :2] == 55).all() and (wide[:, 2 + outs:] == 55).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("tokens,outs,cols", [(1, 300, 4100), (5, 4096, 1000), (8, 2000, 700), (9, 520, 2000), (70, 700, 1000), (513, 1030, 516), (1030, 2060, 200), (2048, 4096, 448), (2300, 5000, 130), (2561, 4097, 520), (300, 40000, 640),
                                             (2817, 3841, 1111)])
def test_linear_of_whole_numbers_is_exact(tokens, outs, cols, transposed, dtype):
    """Sums of whole numbers below 2^24 have no rounding, whatever their order."""
    print("[layers] linear, whole numbers", tokens, outs, cols, transposed, dtype, flush=True)
    x, w = whole(tokens, cols, dtype, 1), whole(cols if transposed else outs, outs if transposed else cols, dtype, 2)
    exact = torch.mm(x.double(), w.double() if transposed else w.double().t())
    assert torch.equal(ogq.ogq_linear(x, w, transposed=transposed), exact.to(dtype))
    y = values(tokens, outs, dtype, 3)
    want = ogq.ogq_linear(x, w, residual=y.clone(), transposed=transposed)
    assert torch.equal(ogq.ogq_linear(x, w, residual=y, transposed=transposed, y=y), want) and torch.equal(y, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("tokens,outs,cols,shift", [(2600, 4200, 576, 0), (1300, 14000, 512, 0), (2600, 4200, 576, 3), (2590, 4100, 601, 0)])
def test_large_linear(tokens, outs, cols, shift, transposed, dtype):
    """More tiles than fit the chip at once, the last ones partly filled; rows that begin anywhere."""
    print("[layers] linear, large", tokens, outs, cols, shift, transposed, dtype, flush=True)
    x = values(tokens, cols, dtype, 1, pad=shift, shift=shift)
    w = values(cols if transposed else outs, outs if transposed else cols, dtype, 2, pad=shift, factor=1.0 / math.sqrt(cols))
    bias, residual = vector(outs, 3), values(tokens, outs, dtype, 4, pad=shift, shift=shift)
    for act, b, r in ((None, None, None), ("gelu", bias, residual)):
        (y, bound), (z, z_bound) = ref.linear(x, w, b, act, r, transposed)
        got, before = ogq.ogq_linear(x, w, b, ACTS[act], r, transposed, keep=True)
        ref.close(got, y, ref.rounded(bound, y, dtype), f"y {act}")
        ref.close(before, z, ref.rounded(z_bound, z, dtype), f"before {act}")
        wide = torch.full((tokens, outs + 8), 55.0, dtype=dtype, device=DEV)
        out = wide[:, :outs]
        out.copy_(values(tokens, outs, dtype, 4) if r is None else r)
        ogq.ogq_linear(x, w, b, ACTS[act], None if r is None else out, transposed, y=out)
        assert torch.equal(out, got) and (wide[:, outs:] == 55).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [2, 40, 200])
def test_linear_of_infinities_and_nan(tokens, dtype):
    x, w = whole(tokens, 90, dtype, 1) + 4, whole(150, 90, dtype, 2) + 4  # no zeros
    x[1, 5], w[7, 5], w[9, 80], x[0, 80] = math.inf, -2.0, math.nan, 0.0
    for transposed in (False, True):
        weight = w.t().contiguous() if transposed else w
        y = ogq.ogq_linear(x, weight, transposed=transposed)
        exact = torch.mm(x.double(), w.double().t())
        assert torch.isnan(y[:, 9]).all()
        keep = torch.ones(150, dtype=torch.bool, device=DEV)
        keep[9] = False
        assert torch.equal(y[:, keep], exact[:, keep].to(dtype))
        assert y[1, 7] == -math.inf and y[1, 8] == math.inf


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_over_nothing(dtype):
    x, w = torch.empty(3, 0, dtype=dtype, device=DEV), torch.empty(5, 0, dtype=dtype, device=DEV)
    bias = vector(5, 1)
    for tokens in (3, 20):
        x = torch.empty(tokens, 0, dtype=dtype, device=DEV)
        for transposed in (False, True):
            y = ogq.ogq_linear(x, w.t() if transposed else w, bias, transposed=transposed)
            assert torch.equal(y, bias.to(dtype).expand(tokens, 5))
    assert ogq.ogq_linear(torch.empty(0, 4, dtype=dtype, device=DEV), torch.empty(5, 4, dtype=dtype, device=DEV)).shape == (0, 5)
    assert ogq.ogq_linear(torch.empty(2, 4, dtype=dtype, device=DEV), torch.empty(0, 4, dtype=dtype, device=DEV)).shape == (2, 0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,outs,pad", [(1, 1, 0), (3, 7, 2), (5, 513, 0), (70, 100, 3), (300, 1000, 0), (2000, 264, 1), (5000, 16, 0)])
def test_linear_backward(tokens, outs, pad, dtype):
    print("[layers] linear backward", tokens, outs, pad, dtype, flush=True)
    dy, before = values(tokens, outs, dtype, 1, pad), values(tokens, outs, dtype, 2, pad, shift=1, factor=2.0)
    chain = (tokens / 16 + 130) * ref.U
    for act in ACTS:
        slope = ref.act(act, before.double())[1]
        off = ref.act_bound(act, before.double(), dtype)[1] * dy.double().abs()
        dz = dy.double() * slope
        got, dbias = ogq.ogq_linear_backward(dy, ACTS[act], None if act is None else before)
        if act is None:
            assert got.data_ptr() == dy.data_ptr()
        else:
            ref.close(got, dz, ref.rounded(off + ref.U * dz.abs(), dz, dtype), f"dz {act}")
        bound = off.sum(0) + chain * dz.abs().sum(0)
        ref.close(dbias, dz.sum(0), ref.rounded(bound, dz.sum(0), torch.float32), f"dbias {act}")
        more = torch.full_like(dbias, 5.0)
        ogq.ogq_linear_backward(dy, ACTS[act], None if act is None else before, dbias=more, accumulate=True)
        assert torch.equal(more, dbias + 5.0)
        if act is not None:
            place = dy.clone()
            assert torch.equal(ogq.ogq_linear_backward(place, ACTS[act], before, dz=place)[0], got)
            place = before.clone()
            assert torch.equal(ogq.ogq_linear_backward(dy, ACTS[act], place, dz=place)[0], got)


# ----------------------------------------------------------------------------------------------------------- embedding
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
@pytest.mark.parametrize("number,vocab,cols,pad", [(1, 1, 1, 0), (5, 3, 7, 2), (64, 10, 8, 0), (127, 2, 33, 0), (128, 1, 100, 1), (200, 1000, 333, 0), (256, 5, 40, 0), (256, 1, 1030, 1), (257, 5, 40, 0), (1024, 50, 64, 0), (1025, 7, 520, 3),
                                                   (3000, 5000, 40, 0), (5000, 3, 24, 0), (40000, 300, 12, 0)])
def test_embedding(number, vocab, cols, pad, ids, dtype):
    print("[layers] embedding", number, vocab, cols, pad, ids, dtype, flush=True)
    gen = torch.Generator(device=DEV).manual_seed(number)
    tokens = torch.randint(-1, vocab + 2, (number,), generator=gen, device=DEV).to(ids)
    table, dy = values(vocab, cols, dtype, 1, pad, shift=pad % 2), values(number, cols, dtype, 2, pad)
    y, bound = ref.embedding(tokens, table, -1.7)
    ref.close(ogq.ogq_embedding_forward(tokens, table, -1.7), y, ref.rounded(bound, y, dtype), "y")
    d, bound = ref.embedding_gradient(tokens, dy, vocab, -1.7)
    got = ogq.ogq_embedding_gradient(tokens, dy, vocab, -1.7)
    ref.close(got, d, ref.rounded(bound, d, torch.float32), "dtable")
    wide = torch.full((vocab, cols + 3), 4.0, device=DEV)
    more = wide[:, 1:1 + cols]
    ogq.ogq_embedding_gradient(tokens, dy, vocab, -1.7, dtable=more, accumulate=True)
    assert torch.equal(more, got + 4.0) and (wide[:, 0] == 4).all() and (wide[:, 1 + cols:] == 4).all()


@pytest.mark.parametrize("number", [100, 256, 2000, 70000])
def test_embedding_gradient_of_whole_numbers_is_exact(number):
    """Few tokens that are frequent, many that are not, some that name no row; int64 beyond 32 bits."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    tokens = torch.cat([torch.randint(0, 4, (number // 2,), generator=gen, device=DEV), torch.randint(0, 900, (number - number // 2,), generator=gen, device=DEV)])
    tokens = tokens[torch.randperm(number, generator=gen, device=DEV)]
    tokens[3], tokens[7], tokens[8] = (1 << 32) + 1, -(1 << 33), 900
    dy = whole(number, 72, torch.bfloat16, 4)
    there = (tokens >= 0) & (tokens < 900)
    exact = torch.zeros(900, 72, dtype=torch.float64, device=DEV).index_add_(0, torch.where(there, tokens, 0), dy.double() * there[:, None])
    assert torch.equal(ogq.ogq_embedding_gradient(tokens, dy, 900).double(), exact)


@pytest.mark.parametrize("vocab,cols", [(20001, 72), (70003, 40), (9000, 1030)])
@pytest.mark.parametrize("number", [1, 64, 65, 256])
def test_embedding_gradient_of_few_tokens_in_a_large_table(number, vocab, cols):
    """One token that stands everywhere but at three places, at the table's end; equal tokens far apart."""
    for dtype in (torch.float32, torch.bfloat16):
        tokens = torch.full((number,), vocab - 1, device=DEV)
        tokens[number // 2], tokens[number // 3], tokens[-1] = 0, vocab // 2, vocab // 2
        dy = whole(number, cols, dtype, 5)
        exact = torch.zeros(vocab, cols, dtype=torch.float64, device=DEV).index_add_(0, tokens, dy.double())
        got = ogq.ogq_embedding_gradient(tokens, dy, vocab)
        assert torch.equal(got.double(), exact)
        ogq.ogq_embedding_gradient(tokens.int(), dy, vocab, -2.0, dtable=got, accumulate=True)
        assert torch.equal(got.double(), -exact)


def test_embedding_over_nothing():
    table = values(5, 6, torch.float32, 1)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    assert ogq.ogq_embedding_forward(none, table).shape == (0, 6)
    assert (ogq.ogq_embedding_gradient(none, table[:0], 5) == 0).all()
    kept = torch.full((5, 6), 3.0, device=DEV)
    ogq.ogq_embedding_gradient(none, table[:0], 5, dtable=kept, accumulate=True)
    assert (kept == 3).all()
    some = torch.tensor([0, 1], device=DEV)
    assert (ogq.ogq_embedding_forward(some, table[:0]) == 0).all()
    assert ogq.ogq_embedding_gradient(some, table[:2], 0).shape == (0, 6)
    assert (ogq.ogq_embedding_gradient(some - 5, table[:2], 5) == 0).all()
    table[1, 2] = math.inf  # (a row that no token names, and one that one names)
    y = ogq.ogq_embedding_forward(torch.tensor([-1, 0, 1], device=DEV), table, 0.0)
    assert (y[0] == 0).all() and (y[1] == 0).all() and torch.isnan(y[2, 2])


# ------------------------------------------------------------------------------------------------------------- distill
def teacher(rows, cols, top, seed, ids=torch.int64):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    places = torch.randint(-1, cols + 1, (rows, top), generator=gen, device=DEV).to(ids)
    return places, 3.0 * torch.randn(rows, top, generator=gen, device=DEV)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,top,pad", [(1, 1, 1, 0), (3, 5, 4, 1), (2, 8, 8, 0), (4, 100, 3, 0), (3, 1000, 1024, 0), (5, 1025, 20, 2), (2, 2048, 1, 0), (3, 4099, 64, 0), (2, 8192, 300, 0),
                                               (2, 8200, 5, 3), (2, 20000, 64, 0), (2, 32769, 100, 1), (2, 65536, 64, 0), (1, 100003, 10, 0), (1, 131072, 64, 0), (1, 140001, 64, 0), (300, 300, 7, 0),
                                               (128, 33001, 9, 0), (129, 33001, 9, 1), (70, 49153, 200, 3), (97, 70001, 30, 1), (97, 131075, 30, 0)])
def test_distill(rows, cols, top, pad, dtype):
    print("[layers] distill", rows, cols, top, pad, dtype, flush=True)
    logits = values(rows, cols, dtype, 1, pad, shift=pad % 2, factor=3.0)
    places, v = teacher(rows, cols, top, 2, torch.int32 if rows % 2 else torch.int64)
    for temperature, row_weight in ((1.0, None), (2.5, vector(rows, 3))):
        (loss, b), (d, bd) = ref.distill(logits, places, v, temperature, row_weight)
        got, dlogits = ogq.ogq_distill_gradient(logits, places, v, temperature, row_weight)
        ref.close(got, loss, ref.rounded(b, loss, torch.float32), "loss")
        ref.close(dlogits, d, ref.rounded(bd, d, dtype), "dlogits")
        assert torch.equal(ogq.ogq_distill_loss(logits, places, v, temperature, row_weight), got)
        place = logits.clone()
        assert torch.equal(ogq.ogq_distill_gradient(place, places, v, temperature, row_weight, dlogits=place)[1], dlogits)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols,times", [(6, 1), (700, 1), (9000, 1), (40000, 1), (140000, 1), (40000, 9), (70001, 9), (140000, 9)])
def test_distill_of_rows_that_are_empty_or_bad(cols, times, dtype):
    """times: the same rows again and again, so many that a row is one workgroup's."""
    rows = 12
    logits = values(rows, cols, dtype, 1)
    places, v = teacher(rows, cols, 5, 2)
    places = places.clamp(0, cols - 1)
    weight = torch.ones(rows, device=DEV)
    places[0] = -1                      # no place
    v[1] = -math.inf                    # no value
    v[2, 3] = -math.inf                 # one place without a share
    v[3, 1] = math.nan
    v[4, 1] = math.inf
    logits[5, 2] = math.nan
    logits[6, 0] = math.inf
    logits[7, 1], places[7] = -math.inf, 4   # a masked logit that the teacher does not have
    logits[8, 1], places[8, 0] = -math.inf, 1  # and one that it has
    weight[9], logits[9, 3] = 0.0, math.nan  # a row that is not looked at
    places[10] = 3                      # one place five times
    logits[11] = -60000.0
    logits[2, 100:] = -math.inf         # all but the row's first logits masked
    (loss, b), (d, bd) = ref.distill(logits, places, v, 1.0, weight)
    logits, places, v, weight = logits.repeat(times, 1), places.repeat(times, 1), v.repeat(times, 1), weight.repeat(times)
    got, dlogits = ogq.ogq_distill_gradient(logits, places, v, 1.0, weight)
    assert torch.equal(ogq.ogq_distill_loss(logits, places, v, 1.0, weight).nan_to_num(), got.nan_to_num())
    for n in range(1, times):
        assert torch.equal(got[n * rows:(n + 1) * rows].nan_to_num(), got[:rows].nan_to_num())
        assert torch.equal(dlogits[n * rows:(n + 1) * rows].nan_to_num(), dlogits[:rows].nan_to_num())
    got, dlogits = got[:rows], dlogits[:rows]
    assert (got[[0, 1, 9]] == 0).all() and (dlogits[[0, 1, 9]] == 0).all()
    for row in (3, 4, 5, 6):
        assert torch.isnan(got[row]) and torch.isnan(dlogits[row]).all(), row
    assert got[8] == math.inf and torch.isfinite(dlogits[8].float()).all() and dlogits[7, 1] == 0
    ref.close(got, loss, ref.rounded(b, loss, torch.float32), "loss")
    ref.close(dlogits, d, ref.rounded(bd, d, dtype), "dlogits")


def test_distill_over_nothing():
    logits = torch.empty(3, 0, device=DEV)
    places, v = torch.zeros(3, 2, dtype=torch.int64, device=DEV), torch.zeros(3, 2, device=DEV)
    loss, d = ogq.ogq_distill_gradient(logits, places, v)
    assert (loss == 0).all() and d.shape == (3, 0)
    logits = values(3, 9, torch.float32, 1)
    loss, d = ogq.ogq_distill_gradient(logits, places[:, :0].contiguous(), v[:, :0].contiguous())
    assert (loss == 0).all() and (d == 0).all()
    assert ogq.ogq_distill_loss(logits[:0], places[:0], v[:0]).shape == (0,)
