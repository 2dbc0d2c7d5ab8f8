"""libogq_layers on the GPU: calls that its documentation allows and that look unlike a training step's: rows that are one and the same, vectors and integers that begin anywhere, results with gaps, results left out."""
import ctypes
import threading

import pytest
import torch

import paper_2002_11082_amd as ogq
from tests.layers_layouts import LINEAR

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
CODE = {torch.float32: ogq.FP32, torch.bfloat16: ogq.BF16, torch.float16: ogq.FP16}


def randn(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)


def shifted(t, by=1):
    """The same values in memory that begins `by` values further."""
    wide = torch.empty(t.numel() + by, dtype=t.dtype, device=DEV)
    wide[by:] = t.reshape(-1)
    return wide[by:].view(t.shape)


def pointer(t):
    return None if t is None else t.data_ptr()


def stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


# ------------------------------------------------------------------------------------------ rows that are one and the same
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [5, 300, 5000, 33000])
def test_norm_of_one_row_again_and_again(cols, dtype):
    x, dy, weight, bias = randn(1, cols, seed=1).to(dtype), randn(1, cols, seed=2).to(dtype), randn(cols, seed=3), randn(cols, seed=4)
    rows = 37
    y, mean, rstd = ogq.ogq_layer_norm_forward(x.expand(rows, cols), weight, bias)
    want = ogq.ogq_layer_norm_forward(x, weight, bias)
    for got, one in zip((y, mean, rstd), want):
        assert torch.equal(got, one.expand_as(got))
    dx, dweight, dbias = ogq.ogq_layer_norm_backward(dy.expand(rows, cols), x.expand(rows, cols), mean, rstd, weight)
    full = ogq.ogq_layer_norm_backward(dy.repeat(rows, 1), x.repeat(rows, 1), mean, rstd, weight)
    for got, one in zip((dx, dweight, dbias), full):
        assert torch.equal(got, one)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("tokens,outs,cols", [(3, 40, 100), (20, 136, 256), (300, 1000, 70), (4096, 4096, 1600), (4096, 4090, 1601)])
def test_linear_of_one_row_again_and_again(tokens, outs, cols, transposed, dtype):
    """x, the weights' rows and the residual, each of them one row."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    whole = lambda *shape: torch.randint(-3, 4, shape, generator=gen, device=DEV).to(dtype)  # noqa: E731
    x, w, residual = whole(tokens, cols), whole(cols if transposed else outs, outs if transposed else cols), whole(1, outs)
    product = lambda x, w: torch.mm(x.double(), w.double() if transposed else w.double().t())  # noqa: E731
    assert torch.equal(ogq.ogq_linear(x[:1].expand(tokens, cols), w, None, None, residual.expand(tokens, outs), transposed),
                       (product(x[:1], w) + residual.double()).to(dtype).expand(tokens, outs))
    same = w[:1].expand(w.shape)
    assert torch.equal(ogq.ogq_linear(x, same, transposed=transposed), product(x, same.contiguous()).to(dtype))


@pytest.mark.parametrize("dtype", TYPES)
def test_the_others_of_one_row_again_and_again(dtype):
    row, rows = randn(1, 700, seed=1).to(dtype), 40
    tokens = torch.randint(0, 9, (rows,), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
    assert torch.equal(ogq.ogq_embedding_forward(tokens, row.expand(9, 700)), row.expand(rows, 700))
    for n in (1, 20):  # in one launch, and sorted
        many = tokens.repeat(n)
        assert torch.equal(ogq.ogq_embedding_gradient(many, row.expand(n * rows, 700), 9), ogq.ogq_embedding_gradient(many, row.repeat(n * rows, 1), 9))
    dz, dbias = ogq.ogq_linear_backward(row.expand(rows, 700), ogq.SILU, row.expand(rows, 700))
    want = ogq.ogq_linear_backward(row.repeat(rows, 1), ogq.SILU, row.repeat(rows, 1))
    assert torch.equal(dz, want[0]) and torch.equal(dbias, want[1])
    places, values = torch.arange(rows * 3, device=DEV).view(rows, 3), randn(rows, 3, seed=3)
    for got, want in zip(ogq.ogq_distill_gradient(row.expand(rows, 700), places, values), ogq.ogq_distill_gradient(row.repeat(rows, 1), places, values)):
        assert torch.equal(got, want)


# --------------------------------------------------------------------------------- vectors and integers that begin anywhere
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(6, 7), (70, 515), (40, 4099), (40, 33001)])
def test_vectors_that_begin_anywhere(rows, cols, dtype):
    x, dy = randn(rows, cols, seed=1).to(dtype), randn(rows, cols, seed=2).to(dtype)
    weight, bias = randn(cols, seed=3), randn(cols, seed=4)
    place = lambda n: torch.empty(n + 3, device=DEV)[3:]  # noqa: E731
    want = ogq.ogq_layer_norm_forward(x, weight, bias)
    got = ogq.ogq_layer_norm_forward(shifted(x), shifted(weight), shifted(bias, 3), mean=place(rows), rstd=place(rows))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    want = ogq.ogq_layer_norm_backward(dy, x, *want[1:], weight)
    got = ogq.ogq_layer_norm_backward(shifted(dy), shifted(x, 2), got[1], got[2], shifted(weight), dweight=place(cols), dbias=place(cols))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    want = ogq.ogq_linear_backward(dy, ogq.GELU, x)
    got = ogq.ogq_linear_backward(shifted(dy), ogq.GELU, shifted(x, 3), dbias=place(cols))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    v, w = randn(rows, 33, seed=5).to(dtype), randn(cols, 33, seed=6).to(dtype)
    assert torch.equal(ogq.ogq_linear(shifted(v), shifted(w, 3), shifted(bias)), ogq.ogq_linear(v, w, bias))


@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
def test_integers_that_begin_anywhere(ids):
    gen = torch.Generator(device=DEV).manual_seed(1)
    table = randn(50, 130, seed=2)
    for number in (100, 1500):
        tokens, dy = torch.randint(-1, 51, (number,), generator=gen, device=DEV).to(ids), randn(number, 130, seed=3)
        assert torch.equal(ogq.ogq_embedding_forward(shifted(tokens), table), ogq.ogq_embedding_forward(tokens, table))
        assert torch.equal(ogq.ogq_embedding_gradient(shifted(tokens), dy, 50), ogq.ogq_embedding_gradient(tokens, dy, 50))
    for cols in (130, 70001):
        logits, places, values, weight = randn(9, cols, seed=4), torch.randint(-1, cols, (9, 7), generator=gen, device=DEV).to(ids), randn(9, 7, seed=5), randn(9, seed=6)
        want = ogq.ogq_distill_gradient(logits, places, values, 1.0, weight)
        got = ogq.ogq_distill_gradient(shifted(logits), shifted(places), shifted(values), 1.0, shifted(weight), loss=torch.empty(10, device=DEV)[1:])
        assert all(torch.equal(a, b) for a, b in zip(got, want))


# ------------------------------------------------------------------------------------------------------ results with gaps
@pytest.mark.parametrize("number", [0, 5, 256, 257, 3000])
@pytest.mark.parametrize("vocab,cols,gap", [(1, 7, 4), (70, 3, 1), (300, 100, 28), (2000, 1030, 5), (5, 16384, 4), (3, 40001, 3)])
def test_a_table_gradient_with_gaps(vocab, cols, gap, number):
    """All of its rows are written, and nothing between them."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    tokens = torch.randint(-1, vocab + 1, (number,), generator=gen, device=DEV)
    dy = torch.randint(-3, 4, (number, cols), generator=gen, device=DEV).bfloat16()
    there = (tokens >= 0) & (tokens < vocab)
    exact = torch.zeros(vocab, cols, dtype=torch.float64, device=DEV).index_add_(0, torch.where(there, tokens, 0), dy.double() * there[:, None])
    wide = torch.full((vocab, cols + gap), 77.0, device=DEV)
    ogq.ogq_embedding_gradient(tokens, dy, vocab, dtable=wide[:, 1:1 + cols])
    assert torch.equal(wide[:, 1:1 + cols].double(), exact)
    assert (wide[:, 0] == 77).all() and (wide[:, 1 + cols:] == 77).all()


def test_gaps_in_a_large_table_cost_little():
    """Short rows are filled together: one at a time they take eighteen times as long as without gaps."""
    vocab, cols = 200000, 16
    tokens, dy = torch.arange(4096, device=DEV) * 17 % vocab, randn(4096, cols, seed=1)
    wide, plain = torch.empty(vocab, cols + 4, device=DEV), torch.empty(vocab, cols, device=DEV)

    def fastest(dtable):
        begin, end, times = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True), []
        for _ in range(6):
            begin.record()
            ogq.ogq_embedding_gradient(tokens, dy, vocab, dtable=dtable)
            end.record()
            end.synchronize()
            times.append(begin.elapsed_time(end))
        return min(times)

    assert fastest(wide[:, :cols]) < 6 * fastest(plain)
    assert torch.equal(wide[:, :cols], plain)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(5, 7), (50, 1000), (30, 5000), (7, 33001), (5, 70003), (100, 140001)])
def test_results_with_gaps(rows, cols, dtype):
    x, dy, weight = randn(rows, cols, seed=1).to(dtype), randn(rows, cols, seed=2).to(dtype), randn(cols, seed=3)

    def into(call):
        wide = torch.full((rows, cols + 5), 77.0, dtype=dtype, device=DEV)
        out = wide[:, 3:3 + cols]
        call(out)
        assert (wide[:, :3] == 77).all() and (wide[:, 3 + cols:] == 77).all()
        return out

    y, mean, rstd = ogq.ogq_layer_norm_forward(x, weight)
    assert torch.equal(into(lambda t: ogq.ogq_layer_norm_forward(x, weight, y=t)), y)
    assert torch.equal(into(lambda t: ogq.ogq_layer_norm_backward(dy, x, mean, rstd, weight, dx=t)), ogq.ogq_layer_norm_backward(dy, x, mean, rstd, weight)[0])
    assert torch.equal(into(lambda t: ogq.ogq_layer_norm_backward(dy, x, mean, rstd, dx=t)), ogq.ogq_layer_norm_backward(dy, x, mean, rstd))
    assert torch.equal(into(lambda t: ogq.ogq_linear_backward(dy, ogq.GELU, x, dz=t)), ogq.ogq_linear_backward(dy, ogq.GELU, x)[0])
    tokens = torch.arange(rows, device=DEV).flip(0)
    assert torch.equal(into(lambda t: ogq.ogq_embedding_forward(tokens, x, y=t)), x.flip(0))
    places, values = torch.randint(-1, cols, (rows, 9), generator=torch.Generator(device=DEV).manual_seed(4), device=DEV), randn(rows, 9, seed=5)
    places[rows // 2] = -1
    assert torch.equal(into(lambda t: ogq.ogq_distill_gradient(x, places, values, dlogits=t)), ogq.ogq_distill_gradient(x, places, values)[1])


# ----------------------------------------------------------------------------------------------------- results left out
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(5, 7), (300, 1000), (9, 70001)])
def test_results_that_the_c_entry_points_leave_out(rows, cols, dtype):
    """The C entry points take NULL where Python makes a tensor."""
    lib, code = ogq.layers_lib(), CODE[dtype]
    x, dy = randn(rows, cols, seed=1).to(dtype), randn(rows, cols, seed=2).to(dtype)
    out = torch.empty_like(x)
    want, mean, rstd = ogq.ogq_layer_norm_forward(x)
    assert lib.ogq_layer_norm_forward(pointer(x), cols, rows, cols, code, None, None, 1e-5, pointer(out), cols, None, None, stream()) == 0
    assert torch.equal(out, want)
    # sums without a weight
    ones = torch.ones(cols, device=DEV)
    sums = [torch.full((cols,), 3.0, device=DEV) for _ in range(2)]
    space = torch.empty(ogq.ogq_layer_norm_backward_workspace(rows, cols, code) + 16, dtype=torch.uint8, device=DEV)
    want = ogq.ogq_layer_norm_backward(dy, x, mean, rstd, ones)
    assert lib.ogq_layer_norm_backward(pointer(dy), cols, pointer(x), cols, rows, cols, code, None, pointer(mean), pointer(rstd), pointer(out), cols, pointer(sums[0]), pointer(sums[1]), 0,
                                       pointer(space), space.numel(), stream()) == 0
    assert torch.equal(out, want[0]) and torch.equal(sums[0], want[1]) and torch.equal(sums[1], want[2])
    # a weight without sums
    weight = randn(cols, seed=3)
    want = ogq.ogq_layer_norm_backward(dy, x, mean, rstd, weight)[0]
    assert lib.ogq_layer_norm_backward(pointer(dy), cols, pointer(x), cols, rows, cols, code, pointer(weight), pointer(mean), pointer(rstd), pointer(out), cols, None, None, 0, None, 0, stream()) == 0
    # (long rows take another kernel: the same formula, of which a 16-bit result may be rounded with a rounding to 32 bits before it or without, so that it is off by a step at most)
    step = torch.finfo(dtype).eps * want.double().abs() + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    assert bool(((out.double() - want.double()).abs() <= step).all())
    # dz alone
    want = ogq.ogq_linear_backward(dy, ogq.GELU_TANH, x)[0]
    assert lib.ogq_linear_backward(pointer(dy), cols, rows, cols, code, ogq.GELU_TANH, pointer(x), cols, pointer(out), cols, None, 0, None, 0, stream()) == 0
    assert torch.equal(out, want)
    # a gradient without the loss
    places, values = torch.arange(rows * 2, device=DEV).view(rows, 2) % cols, randn(rows, 2, seed=4)
    space = torch.empty(ogq.ogq_distill_workspace(rows, cols, code, 2) + 16, dtype=torch.uint8, device=DEV)
    want = ogq.ogq_distill_gradient(x, places, values)[1]
    assert lib.ogq_distill_gradient(pointer(x), cols, rows, cols, code, pointer(places), ogq.INT64, pointer(values), 2, 1.0, None, None, pointer(out), cols, pointer(space), space.numel(), stream()) == 0
    assert torch.equal(out, want)


# ------------------------------------------------------------------------------------------------------------ workspaces
class Space:
    """A workspace of exactly the bytes that are asked for, between others that stay as they are; its contents are NaN at first."""

    def __init__(self, size):
        self.whole = torch.full((16 * 1024 + (size + 15) // 16 * 16 + 16 * 1024,), 0xFF, dtype=torch.uint8, device=DEV)
        self.size, self.space = size, self.whole[16 * 1024:16 * 1024 + size]

    def unharmed(self):
        return bool((self.whole[:16 * 1024] == 0xFF).all()) and bool((self.whole[16 * 1024 + self.size:] == 0xFF).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_workspaces_of_just_the_right_size(dtype):
    code = CODE[dtype]
    for rows, cols in ((3, 2), (70, 7), (5, 300), (3000, 100), (2100, 515), (700, 4099), (520, 9001), (40, 33001), (3, 40001), (300, 17000)):
        print("[layers] workspaces", rows, cols, dtype, flush=True)
        x, dy, weight = randn(rows, cols, seed=1).to(dtype), randn(rows, cols, seed=2).to(dtype), randn(cols, seed=3)
        _, mean, rstd = ogq.ogq_layer_norm_forward(x, weight)
        space = Space(ogq.ogq_layer_norm_backward_workspace(rows, cols, code))
        got, want = ogq.ogq_layer_norm_backward(dy, x, mean, rstd, weight, workspace=space.space), ogq.ogq_layer_norm_backward(dy, x, mean, rstd, weight)
        assert space.unharmed() and all(torch.equal(a, b) for a, b in zip(got, want))
        space = Space(ogq.ogq_linear_backward_workspace(rows, cols, code))
        got, want = ogq.ogq_linear_backward(dy, ogq.GELU, x, workspace=space.space), ogq.ogq_linear_backward(dy, ogq.GELU, x)
        assert space.unharmed() and all(torch.equal(a, b) for a, b in zip(got, want))
        places, values = torch.arange(rows * 5, device=DEV).view(rows, 5) % cols, randn(rows, 5, seed=4)
        space = Space(ogq.ogq_distill_workspace(rows, cols, code, 5))
        got, want = ogq.ogq_distill_gradient(x, places, values, workspace=space.space), ogq.ogq_distill_gradient(x, places, values)
        assert space.unharmed() and all(torch.equal(a, b) for a, b in zip(got, want))
        tokens = torch.arange(rows, device=DEV) * 7919 % 50
        space = Space(ogq.ogq_embedding_gradient_workspace(rows, 50, cols))
        got, want = ogq.ogq_embedding_gradient(tokens, dy, 50, workspace=space.space), ogq.ogq_embedding_gradient(tokens, dy, 50)
        assert space.unharmed() and torch.equal(got, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transposed", [False, True])
def test_workspaces_of_linear_layers(transposed, dtype):
    for tokens, outs, cols, _ in LINEAR + [(3, 300, 5000, 0), (8, 1001, 2000, 0), (256, 4096, 2100, 0)]:
        x, w = randn(tokens, cols, seed=1).to(dtype), randn(cols if transposed else outs, outs if transposed else cols, seed=2).to(dtype)
        space = Space(ogq.ogq_linear_workspace(tokens, outs, cols, CODE[dtype], transposed))
        got = ogq.ogq_linear(x, w, transposed=transposed, workspace=space.space)
        assert space.unharmed() and torch.equal(got, ogq.ogq_linear(x, w, transposed=transposed)), (tokens, outs, cols)


def test_calls_of_several_launches_in_graphs():
    """Two graphs of calls that use a workspace, replayed in turn with other inputs and eager calls between them."""
    shapes = {"x": (40, 33001), "dy": (40, 33001), "a": (70, 4100), "w": (3000, 4100), "e": (3000, 520), "z": (9, 70001)}

    def inputs(seed):
        t = {name: randn(*shape, seed=seed + n) for n, (name, shape) in enumerate(shapes.items())}
        gen = torch.Generator(device=DEV).manual_seed(seed)
        t["tokens"] = torch.randint(-1, 60, (3000,), generator=gen, device=DEV)
        t["places"], t["values"] = torch.randint(-1, 70001, (9, 6), generator=gen, device=DEV), randn(9, 6, seed=seed + 20)
        t["x"][::3] += 1.0e5  # (rows far from zero)
        return t

    def calls(t):
        y, mean, rstd = ogq.ogq_layer_norm_forward(t["x"])
        weight = t["dy"][0].abs() + 0.5
        return [y, *ogq.ogq_layer_norm_backward(t["dy"], t["x"], mean, rstd, weight), ogq.ogq_linear(t["a"], t["w"], None, ogq.GELU), ogq.ogq_linear_backward(t["e"])[1],
                ogq.ogq_embedding_gradient(t["tokens"], t["e"], 60), *ogq.ogq_distill_gradient(t["z"], t["places"], t["values"])]

    static = inputs(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(static)
    torch.cuda.current_stream().wait_stream(side)
    graphs, results = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results.append(calls(static))
        graphs.append(graph)
    for n in range(6):
        new = inputs(100 * n + 7)
        for name, t in static.items():
            t.copy_(new[name])
        graphs[n % 2].replay()
        eager = calls(static)
        torch.cuda.synchronize()
        for got, want in zip(results[n % 2], eager):
            assert torch.equal(got, want), n


def test_calls_at_the_same_time():
    """Two threads with a stream each: the calls have nothing in common."""
    def inputs(seed):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        return (randn(60, 33001, seed=seed), randn(33001, seed=seed + 1), randn(70, 4100, seed=seed + 2).bfloat16(), randn(3000, 4100, seed=seed + 3).bfloat16(),
                torch.randint(-1, 50, (3000,), generator=gen, device=DEV), randn(3000, 400, seed=seed + 4), torch.randint(-1, 33001, (60, 8), generator=gen, device=DEV), randn(60, 8, seed=seed + 5))

    def calls(x, weight, a, w, tokens, e, places, values):
        y, mean, rstd = ogq.ogq_layer_norm_forward(x, weight)
        return [y, *ogq.ogq_layer_norm_backward(y, x, mean, rstd, weight), ogq.ogq_linear(a, w, None, ogq.SILU), ogq.ogq_linear(w, a),
                ogq.ogq_embedding_gradient(tokens, e, 50), *ogq.ogq_distill_gradient(x, places, values)]

    given = [inputs(1), inputs(50)]
    want = [calls(*t) for t in given]
    torch.cuda.synchronize()
    wrong = []

    def run(n):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(10):
                got = calls(*given[n])
                torch.cuda.current_stream().synchronize()
                wrong.extend(i for i, (a, b) in enumerate(zip(got, want[n])) if not torch.equal(a, b))

    threads = [threading.Thread(target=run, args=(n,)) for n in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not any(t.is_alive() for t in threads) and wrong == []
