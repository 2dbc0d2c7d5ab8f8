"""The layers around the tensors held in groups, from a program's tokens to its loss, as cases that can be timed and compared.

A program that trains with the package has tokens that become rows of a table, layers that normalise them and multiply them with weights, and a teacher whose
largest logits it learns.  A case is one of

  op       "norm": layer norm over the columns, with a weight and a bias in fp32 where `affine`; its backward pass too where `train`: the gradient of the
           inputs, and those of weight and bias, sums over all rows
           "linear": act(x W^T + bias) + residual, a layer's forward pass; what went into the activation is left for the backward pass where `train`
           "linear_backward": what a layer's backward pass makes of the gradient of act(x W^T + bias): that of what went into the activation, its sums over
           the tokens (the bias' gradient), and its products with W (the inputs' gradient)
           "embedding": rows of a table by tokens, times a scale; where `train` also the table's gradient, the scaled sums of the gradients of equal tokens
           "distill": the divergence of a student's distribution from a teacher's, of which a few logits and their places are known; where `train`
           also the gradient of the student's logits

for `rows` rows (tokens), `cols` columns (inputs, the table's width, the logits of a row), `outs` outputs of a layer, a table of `vocab` rows, `top` teacher's
logits of a row, in `dtype`; `pad` values lie between the end of a row and the next one.  Tokens and places of logits are `ids` integers; those that are not in the
table or the row stand for none (a sequence that was padded, a shorter list of a teacher's).  Layers are those of the package's benchmark (the fully connected
layers of VGG-19, 25088 to 4096 to 4096 to 1000, and its batch of 256) and of a block of width 4096 with a hidden width of 16384.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-5


def _case(name, op, rows, cols, dtype, outs=0, vocab=0, top=0, act="", affine=True, bias=True, residual=False, train=True, temperature=1.0, ids="int64", pad=0):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "outs": outs, "vocab": vocab, "top": top, "dtype": dtype, "act": act, "affine": affine,
            "bias": bias, "residual": residual, "train": train, "temperature": temperature, "ids": ids, "pad": pad}


def listed():
    return [
        # One token that is answered: a launch and a chain of latencies.
        _case("norm_token", "norm", 1, 4096, "bf16", train=False),
        # The norm in front of a block in a training step, 8192 tokens of width 4096, forward and backward.
        _case("norm_block", "norm", 8192, 4096, "bf16"),
        # A view into a wider tensor, rows that start anywhere, in 32 bits: the sums over the rows weigh most.
        _case("norm_view", "norm", 1237, 1001, "fp32", pad=7),
        # One token through the block's first linear layer: the weights are read once, nothing else counts.
        _case("linear_token", "linear", 1, 4096, "bf16", outs=16384, act="silu", train=False),
        # The block's first linear layer in a training step, the largest product of a forward pass.
        _case("linear_block", "linear", 8192, 4096, "bf16", outs=16384, act="gelu"),
        # The first fully connected layer of VGG-19, its batch of 256, in 32 bits: a long sum for few outputs.
        _case("linear_batch", "linear", 256, 25088, "fp32", outs=4096, act="relu"),
        # A few sequences served together through a layer that adds to what went around it, odd in every direction.
        _case("linear_residual", "linear", 37, 1001, "fp16", outs=2589, residual=True, train=False, pad=3),
        # The backward pass of the block's second layer over half of a step's tokens: its gradient from 4096 outputs to 16384 inputs.
        _case("backward_block", "linear_backward", 4096, 16384, "bf16", outs=4096, act="gelu_tanh"),
        # A step's tokens: 16384 of a table of 32768 rows of width 4096, some far more frequent than others, some padded.
        _case("embedding_block", "embedding", 16384, 4096, "bf16", vocab=32768),
        # A few sequences of a small table, odd in every direction, in 32 bits.
        _case("embedding_few", "embedding", 200, 333, "fp32", vocab=1000, ids="int32"),
        # 4096 tokens learn a teacher's 64 largest logits of 32768.
        _case("distill_block", "distill", 4096, 32768, "bf16", top=64, temperature=2.0),
        # A few tokens against a large table in fp16 whose rows start anywhere: one row's latency.
        _case("distill_wide", "distill", 61, 131071, "fp16", top=100, ids="int32", pad=2),
    ]


def _log(rng, low, high):
    low, high = min(low, high), max(low, high)
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    """One more case: any type, one row to many, widths that no power of two divides."""
    op = rng.choice(("norm", "linear", "linear", "linear_backward", "embedding", "distill"))
    dtype = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    pad = rng.choice((0, 0, 0, 1, 8, 24))
    train = rng.random() < 0.7
    ids = rng.choice(("int32", "int64"))
    even = rng.random() < 0.5
    if op == "norm":
        cols = _log(rng, 32, 16384)
        cols = max(32, cols // 32 * 32) if even else cols
        case = _case("", op, _log(rng, 1, min(16384, 33554432 // cols)), cols, dtype, affine=rng.random() < 0.8, train=train, pad=pad)
    elif op == "linear" or op == "linear_backward":
        cols, outs = _log(rng, 16, 25088), _log(rng, 16, 16384)
        if even:
            cols, outs = max(32, cols // 32 * 32), max(32, outs // 32 * 32)
        rows = rng.choice((1, rng.randint(2, 64), _log(rng, 1, 16384), _log(rng, 64, 16384)))
        rows = min(rows, max(1, (549755813888 if dtype != "fp32" else 137438953472) // (cols * outs)))
        act = rng.choice(("", "relu", "gelu", "gelu_tanh", "silu"))
        case = _case("", op, rows, cols, dtype, outs=outs, act=act, bias=rng.random() < 0.8, residual=op == "linear" and rng.random() < 0.4, train=train, pad=pad)
    elif op == "embedding":
        cols, vocab = _log(rng, 16, 8192), _log(rng, 64, 131072)
        cols = max(16, cols // 16 * 16) if even else cols
        vocab = min(vocab, 134217728 // cols)
        rows = _log(rng, 1, min(32768, 67108864 // cols))
        case = _case("", op, rows, cols, dtype, vocab=vocab, train=train, ids=ids, pad=pad)
    else:
        cols = _log(rng, 256, 131072)
        cols = cols // 64 * 64 if even else cols
        rows = _log(rng, 1, min(8192, 134217728 // cols))
        case = _case("", op, rows, cols, dtype, top=_log(rng, 1, 128), temperature=rng.choice((1.0, 1.0, 2.0, 4.0)), train=train, ids=ids, pad=pad)
    del case["name"]
    return case


def _act(name, x):
    """An activation and its derivative."""
    if name == "":
        return x, torch.ones_like(x)
    if name == "relu":
        on = (x > 0.0).float()
        return x * on, on
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-x))
        return x * s, s * (1.0 + x * (1.0 - s))
    if name == "gelu":
        p = 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5)))
        return x * p, p + x * torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2.0 * math.pi))
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (x + 0.044715 * x * x * x))
    return 0.5 * x * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * x * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * x * x)


def _wide(values, dtype, pad):
    """Values as rows of a tensor that has `pad` more values in each."""
    wide = torch.empty(values.shape[0], values.shape[1] + pad, dtype=dtype, device="cuda")
    x = wide[:, :values.shape[1]]
    x.copy_(values)
    return x


def _activations(gen, rows, cols, dtype, pad, factor=1.0):
    """Activations: every channel of its own size and offset, a few of them large, and rows of zeros where a sequence was padded."""
    size = torch.exp(0.5 * torch.randn(cols, generator=gen, device="cuda"))
    size = torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.003, 20.0 * size, size)
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    x.add_(0.3 * torch.randn(cols, generator=gen, device="cuda")).mul_(size * factor)
    if rows > 16:
        x[torch.rand(rows, generator=gen, device="cuda") < 0.02] = 0.0
    return _wide(x, dtype, pad)


def prepare(case, seed):
    """The tensors that a program has in hand."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, rows, cols, outs, vocab, top, pad = (case[k] for k in ("op", "rows", "cols", "outs", "vocab", "top", "pad"))
    dtype, ids = DTYPES[case["dtype"]], torch.int32 if case["ids"] == "int32" else torch.int64
    s = {"case": case, "dtype": dtype}
    if op == "norm":
        s["x"] = _activations(gen, rows, cols, dtype, pad)
        s["weight"] = 1.0 + 0.2 * torch.randn(cols, generator=gen, device="cuda") if case["affine"] else None
        s["bias"] = 0.2 * torch.randn(cols, generator=gen, device="cuda") if case["affine"] else None
        s["dy"] = _activations(gen, rows, cols, dtype, pad, 1e-2) if case["train"] else None
    elif op == "linear" or op == "linear_backward":
        s["weight"] = _wide(torch.randn(outs, cols, generator=gen, device="cuda") / math.sqrt(cols), dtype, pad)
        s["bias"] = 0.2 * torch.randn(outs, generator=gen, device="cuda") if case["bias"] else None
        if op == "linear":
            s["x"] = _activations(gen, rows, cols, dtype, pad)
            s["residual"] = _activations(gen, rows, outs, dtype, pad) if case["residual"] else None
        else:
            s["before"] = _activations(gen, rows, outs, dtype, pad) if case["act"] else None
            s["dy"] = _activations(gen, rows, outs, dtype, pad, 1e-1)
    elif op == "embedding":
        # one over the rank: the most frequent token is every tenth or so
        rank = torch.exp(torch.rand(rows, generator=gen, device="cuda", dtype=torch.float64) * math.log(vocab)).long().clamp(max=vocab) - 1
        tokens = (rank * 7919 + seed % vocab) % vocab
        s["tokens"] = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.03, -1, tokens).to(ids)
        s["table"] = _wide(torch.randn(vocab, cols, generator=gen, device="cuda") / math.sqrt(cols), dtype, pad)
        s["dy"] = _activations(gen, rows, cols, dtype, pad, 1e-2) if case["train"] else None
        s["scale"] = math.sqrt(cols)
    else:
        logits = 2.0 * torch.randn(rows, cols, generator=gen, device="cuda")
        places = torch.randint(0, cols, (rows, top), generator=gen, device="cuda")
        values = 8.0 + 2.0 * torch.randn(rows, top, generator=gen, device="cuda")
        logits.scatter_(1, places, values + torch.randn(rows, top, generator=gen, device="cuda"))
        places = torch.where(torch.rand(rows, top, generator=gen, device="cuda") < 0.05, -1, places)
        if rows > 16:
            places[torch.rand(rows, generator=gen, device="cuda") < 0.02] = -1
        s["logits"], s["places"], s["values"] = _wide(logits, dtype, pad), places.to(ids), values
        # the mean over the tokens, and the factor that keeps a step's gradients in fp16
        s["row_weight"] = torch.full((rows,), (65536.0 if dtype == torch.float16 else 1.0) / rows, device="cuda")
    return s


def _plain_norm(s):
    c, dtype = s["case"], s["dtype"]
    x = s["x"].float()
    mean = x.sum(1, keepdim=True) / c["cols"]
    off = x - mean
    rstd = 1.0 / torch.sqrt((off * off).sum(1, keepdim=True) / c["cols"] + EPS)
    unit = off * rstd
    y = unit if s["weight"] is None else unit * s["weight"] + s["bias"]
    out = {"y": y.to(dtype)}
    if c["train"]:
        dy = s["dy"].float()
        g = dy if s["weight"] is None else dy * s["weight"]
        along = (g * unit).sum(1, keepdim=True) / c["cols"]
        out["dx"] = (rstd * (g - g.sum(1, keepdim=True) / c["cols"] - unit * along)).to(dtype)
        if s["weight"] is not None:
            out["dweight"], out["dbias"] = (dy * unit).sum(0), dy.sum(0)
    return out


def _plain_linear(s):
    c, dtype = s["case"], s["dtype"]
    z = s["x"].float() @ s["weight"].float().t()
    if s["bias"] is not None:
        z = z + s["bias"]
    y = _act(c["act"], z)[0]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(dtype), "before": z.to(dtype)} if c["train"] else {"y": y.to(dtype)}


def _plain_linear_backward(s):
    c, dtype = s["case"], s["dtype"]
    dz = s["dy"].float()
    if c["act"]:
        dz = dz * _act(c["act"], s["before"].float())[1]
    # (as the layer's other gradients read it, in its type)
    held = dz.to(dtype)
    return {"dz": held, "dbias": dz.sum(0), "dx": (held.float() @ s["weight"].float()).to(dtype)}


def _plain_embedding(s):
    c, dtype = s["case"], s["dtype"]
    tokens = s["tokens"].long()
    there = ((tokens >= 0) & (tokens < c["vocab"])).unsqueeze(1)
    at = torch.where(there[:, 0], tokens, 0)
    out = {"y": (torch.where(there, s["table"][at].float(), 0.0) * s["scale"]).to(dtype)}
    if c["train"]:
        dy = torch.where(there, s["dy"].float() * s["scale"], 0.0)
        out["dtable"] = torch.zeros(c["vocab"], c["cols"], device=dy.device).index_add_(0, at, dy)
    return out


def _plain_distill(s):
    c, dtype = s["case"], s["dtype"]
    tau = c["temperature"]
    z, places = s["logits"].float() / tau, s["places"].long()
    there = (places >= 0) & (places < c["cols"])
    some = there.any(1, keepdim=True)
    at = torch.where(there, places, 0)
    v = torch.where(there, s["values"] / tau, float("-inf"))
    e = torch.where(there, torch.exp(v - torch.where(some, v.amax(1, keepdim=True), 0.0)), 0.0)
    p = e / torch.where(some, e.sum(1, keepdim=True), 1.0)
    z = z - z.amax(1, keepdim=True)
    q = torch.exp(z)
    total = q.sum(1, keepdim=True)
    log_p, log_q = torch.log(torch.where(p > 0.0, p, 1.0)), z.gather(1, at) - torch.log(total)
    weight = s["row_weight"]
    out = {"loss": weight * tau * tau * torch.where(p > 0.0, p * (log_p - log_q), 0.0).sum(1)}
    if c["train"]:
        dz = (q / total * some).scatter_add_(1, at, -p) * (weight * tau).unsqueeze(1)
        out["dlogits"] = dz.to(dtype)
    return out


PLAIN = {"norm": _plain_norm, "linear": _plain_linear, "linear_backward": _plain_linear_backward, "embedding": _plain_embedding, "distill": _plain_distill}


def run(s):
    if not own:
        return PLAIN[s["case"]["op"]](s)
    import paper_2002_11082_amd as ogq
    c = s["case"]
    act = {"": None, "relu": ogq.RELU, "silu": ogq.SILU, "gelu": ogq.GELU, "gelu_tanh": ogq.GELU_TANH}[c["act"]]
    if c["op"] == "norm":
        y, mean, rstd = ogq.ogq_layer_norm_forward(s["x"], s["weight"], s["bias"], EPS)
        if not c["train"]:
            return {"y": y}
        if s["weight"] is None:
            return {"y": y, "dx": ogq.ogq_layer_norm_backward(s["dy"], s["x"], mean, rstd)}
        dx, dweight, dbias = ogq.ogq_layer_norm_backward(s["dy"], s["x"], mean, rstd, s["weight"])
        return {"y": y, "dx": dx, "dweight": dweight, "dbias": dbias}
    if c["op"] == "linear":
        if not c["train"]:
            return {"y": ogq.ogq_linear(s["x"], s["weight"], s["bias"], act, s["residual"])}
        y, before = ogq.ogq_linear(s["x"], s["weight"], s["bias"], act, s["residual"], keep=True)
        return {"y": y, "before": before}
    if c["op"] == "linear_backward":
        dz, dbias = ogq.ogq_linear_backward(s["dy"], act, s["before"])
        return {"dz": dz, "dbias": dbias, "dx": ogq.ogq_linear(dz, s["weight"], transposed=True)}
    if c["op"] == "embedding":
        out = {"y": ogq.ogq_embedding_forward(s["tokens"], s["table"], s["scale"])}
        if c["train"]:
            out["dtable"] = ogq.ogq_embedding_gradient(s["tokens"], s["dy"], c["vocab"], s["scale"])
        return out
    if not c["train"]:
        return {"loss": ogq.ogq_distill_loss(s["logits"], s["places"], s["values"], c["temperature"], s["row_weight"])}
    loss, dlogits = ogq.ogq_distill_gradient(s["logits"], s["places"], s["values"], c["temperature"], s["row_weight"])
    return {"loss": loss, "dlogits": dlogits}


def work(case):
    rows, cols, outs, vocab, top = (case[k] for k in ("rows", "cols", "outs", "vocab", "top"))
    size, wide = 4 if case["dtype"] == "fp32" else 2, 4 if case["ids"] == "int32" else 8
    if case["op"] == "norm":  # x in, y out; with the gradient of y in, that of x out; weight and bias, and their gradients
        tensors, vectors = (4, 4) if case["train"] else (2, 2)
        return {"bytes": tensors * rows * cols * size + (4 * vectors * cols if case["affine"] else 0), "flops": (20 if case["train"] else 8) * rows * cols}
    if case["op"] == "linear":
        results = 1 + case["train"] + case["residual"]
        return {"bytes": (rows * cols + outs * cols + results * rows * outs) * size + (4 * outs if case["bias"] else 0), "flops": 2 * rows * outs * cols}
    if case["op"] == "linear_backward":
        return {"bytes": (rows * cols + outs * cols + (3 if case["act"] else 2) * rows * outs) * size + 4 * outs, "flops": 2 * rows * outs * cols}
    if case["op"] == "embedding":  # the rows that tokens name, at most all of the table; the gradient of every row
        most = min(rows, vocab)
        return {"bytes": (most + rows) * cols * size + rows * wide + ((rows * size + vocab * 4) * cols if case["train"] else 0), "flops": (2 if case["train"] else 1) * rows * cols}
    return {"bytes": (2 if case["train"] else 1) * rows * cols * size + rows * (top * (wide + 4) + 8), "flops": (6 if case["train"] else 4) * rows * cols}


# ----------------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ----------------------------------------------------------------------------------------------------------------------
def _exact_act(name, x):
    if name == "":
        return x, torch.ones_like(x)
    if name == "relu":
        return x.clamp(min=0.0), (x > 0.0).double()
    if name == "silu":
        s = torch.sigmoid(x)
        return x * s, s + x * s * torch.sigmoid(-x)
    if name == "gelu":
        p = 0.5 * torch.erfc(-x / math.sqrt(2.0))
        return x * p, p + x * torch.exp(-x * x / 2.0) / math.sqrt(2.0 * math.pi)
    u = 2.0 * math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3)  # (1 + tanh(u / 2)) / 2 = 1 / (1 + exp(-u))
    s = torch.sigmoid(u)
    return x * s, s + x * s * torch.sigmoid(-u) * 2.0 * math.sqrt(2.0 / math.pi) * (1.0 + 3.0 * 0.044715 * x * x)


def _exact_norm(s):
    x, c = s["x"].double(), s["case"]
    variance, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    deviation = (variance + EPS).sqrt()
    y = (x - mean) / deviation
    out = {"y": y if s["weight"] is None else torch.addcmul(s["bias"].double(), y, s["weight"].double())}
    if c["train"]:
        # the Jacobian of a row, (1 - 1/n - y y^T / n) / deviation, times the gradient
        dy = s["dy"].double()
        g = dy if s["weight"] is None else dy * s["weight"].double()
        out["dx"] = (g - g.mean(1, keepdim=True) - y * (g * y).mean(1, keepdim=True)) / deviation
        if s["weight"] is not None:
            ones = torch.ones(1, c["rows"], dtype=torch.float64, device=x.device)
            out["dweight"], out["dbias"] = (ones @ (dy * y))[0], (ones @ dy)[0]
    return out


def _exact_linear(s):
    z = torch.mm(s["x"].double(), s["weight"].double().t())
    if s["bias"] is not None:
        z += s["bias"].double()
    y = _exact_act(s["case"]["act"], z)[0]
    if s["residual"] is not None:
        y = y + s["residual"].double()
    return {"y": y, "before": z} if s["case"]["train"] else {"y": y}


def _exact_linear_backward(s):
    dz = s["dy"].double()
    if s["case"]["act"]:
        dz = dz * _exact_act(s["case"]["act"], s["before"].double())[1]
    return {"dz": dz, "dbias": (torch.ones(1, dz.shape[0], dtype=torch.float64, device=dz.device) @ dz)[0], "dx": torch.mm(dz, s["weight"].double())}


def _exact_embedding(s):
    c, tokens = s["case"], s["tokens"].long()
    there = (tokens >= 0) & (tokens < c["vocab"])
    y = torch.zeros(c["rows"], c["cols"], dtype=torch.float64, device=tokens.device)
    y[there] = s["table"].double()[tokens[there]] * s["scale"]
    out = {"y": y}
    if c["train"]:
        # differences of a running sum over the gradients in the tokens' order
        order = torch.argsort(torch.where(there, tokens, c["vocab"]))
        running = torch.cumsum(s["dy"].double()[order] * s["scale"], 0)
        running = torch.cat([torch.zeros_like(running[:1]), running])
        ends = torch.searchsorted(torch.where(there, tokens, c["vocab"])[order], torch.arange(c["vocab"], device=tokens.device), right=True)
        starts = torch.cat([torch.zeros_like(ends[:1]), ends[:-1]])
        out["dtable"] = running[ends] - running[starts]
    return out


def _exact_distill(s):
    c, tau, places = s["case"], s["case"]["temperature"], s["places"].long()
    log_q = torch.log_softmax(s["logits"].double() / tau, 1)
    there = (places >= 0) & (places < c["cols"])
    values = torch.where(there, s["values"].double() / tau, float("-inf"))
    log_p = values - torch.logsumexp(values, 1, keepdim=True)
    log_p = torch.where(there, log_p, 0.0)
    p = torch.where(there, torch.exp(log_p), 0.0)
    weight = s["row_weight"].double()
    out = {"loss": weight * tau ** 2 * (p * (log_p - log_q.gather(1, torch.where(there, places, 0)))).sum(1)}
    if c["train"]:
        target = torch.zeros_like(log_q).scatter_add_(1, torch.where(there, places, 0), p)
        out["dlogits"] = (torch.exp(log_q) * there.any(1, keepdim=True) - target) * (weight * tau).unsqueeze(1)
    return out


EXACT = {"norm": _exact_norm, "linear": _exact_linear, "linear_backward": _exact_linear_backward, "embedding": _exact_embedding, "distill": _exact_distill}


def exact(case, seed):
    return EXACT[case["op"]](prepare(case, seed))
