"""The operators of a training step whose weights AdamW steps, as cases that can be timed and compared: norms and embedding.

A case is a dict of plain values. Its "call" says which operator it runs:

  norm            layer norm or RMS norm, with the residual stream's addition (`meq.layer_norm`, `meq.rms_norm`)
  norm_grad       its backward pass: the gradients of the input, the weight and the bias (`meq.layer_norm_grad`,
                  `meq.rms_norm_grad`)
    kind          "layer" (a mean, a bias) or "rms"
    rows, cols    tokens and width; dtype: of the tokens; weight: type of the weight, the bias and their gradients
    residual      norm: the tokens are added to a residual stream first, which is written too; norm_grad: the
                  stream's own gradient is added to the input's
    pad, shift    columns of padding after each row, and elements by which the buffers' starts are moved
  embedding       rows of the table for the tokens, scaled (`meq.embedding`)
  embedding_grad  the table's gradient, every row of it (`meq.embedding_grad`)
    tokens, vocab, cols    tokens of the batch, rows and width of the table
    table, dtype  types of the table (or of its gradient) and of the tokens' vectors (or of their gradients)
    masked        share of the tokens that are padding (negative)
    tied          embedding_grad: added to what the table's gradient holds already (a head that shares the table)
    pad, shift    as above, of the tokens' vectors
"""
import math
import random

import torch

own = False

EPS = {"layer": 1e-5, "rms": 1e-6}
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}


# -------------------------------------------------------------------- cases
def _norm(call, kind, rows, cols, dtype="bf16", weight="fp32", residual=False, pad=0, shift=0, name=None):
    c = {"call": call, "kind": kind, "rows": rows, "cols": cols, "dtype": dtype, "weight": weight, "residual": residual, "pad": pad,
         "shift": shift}
    return c if name is None else dict(c, name=name)


def _embed(call, tokens, vocab, cols, table="fp32", dtype="bf16", masked=0.1, tied=False, pad=0, shift=0, name=None):
    c = {"call": call, "tokens": tokens, "vocab": vocab, "cols": cols, "table": table, "dtype": dtype, "masked": masked, "pad": pad,
         "shift": shift}
    if call == "embedding_grad":
        c["tied"] = tied
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # One decoding step of 16 candidates through a 130M model: the smallest call, where latency counts.
        _norm("norm", "rms", 16, 768, residual=True, name="rms norm 16 candidates"),
        # Activations in fp32 and an ordinary batch, mean and bias.
        _norm("norm", "layer", 8192, 2048, dtype="fp32", name="layer norm 8192 x 2048 fp32"),
        # An odd width: every row starts elsewhere in its 16 bytes.
        _norm("norm", "layer", 6001, 1025, residual=True, name="layer norm odd width"),
        # A large batch of a 7B-class model, in the residual stream.
        _norm("norm", "rms", 32768, 4096, weight="bf16", residual=True, name="rms norm 32768 x 4096"),
        # The backward pass over one short answer in fp32.
        _norm("norm_grad", "rms", 24, 768, dtype="fp32", residual=True, name="rms norm grad short answer"),
        # An ordinary minibatch of a 350M model under a loss scale in fp16, with the bias's gradient.
        _norm("norm_grad", "layer", 8192, 1024, dtype="fp16", name="layer norm grad 8192 x 1024"),
        # The large batch of the 7B-class model, everything in bf16.
        _norm("norm_grad", "rms", 32768, 4096, weight="bf16", residual=True, name="rms norm grad 32768 x 4096"),
        # The tokens of one decoding step.
        _embed("embedding", 16, 32000, 768, table="bf16", masked=0.0, name="embedding 16 tokens"),
        # A packed batch from an fp32 table into bf16 vectors.
        _embed("embedding", 65536, 32000, 2048, name="embedding 65536 tokens"),
        # One short answer: nearly every row of the gradient is zero, and all are written.
        _embed("embedding_grad", 24, 32000, 768, masked=0.0, name="embedding grad short answer"),
        # An ordinary minibatch; table shared with the head, odd width and vocabulary.
        _embed("embedding_grad", 6000, 50001, 1001, table="fp32", dtype="fp16", masked=0.3, tied=True, name="embedding grad odd tied"),
        # A packed batch of a 7B-class width over a large vocabulary, the gradient in bf16.
        _embed("embedding_grad", 65536, 151936, 4096, table="bf16", name="embedding grad large vocabulary"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    n = _log_uniform(rng, lo, hi)
    return 64 * max(1, n // 64) if rng.random() < 0.6 else n


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    call = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "norm_grad", "embedding", "embedding_grad", "embedding_grad"])
    while True:
        opts = {"dtype": rng.choice(["bf16", "bf16", "bf16", "fp16", "fp32"]), "pad": rng.choice([0, 0, 0, 1, 8, 64]),
                "shift": rng.choice([0, 0, 0, 0, 1, 3])}
        if call.startswith("norm"):
            c = _norm(call, rng.choice(["layer", "rms"]), _log_uniform(rng, 1, 60000), _width(rng, 32, 16384),
                      weight=rng.choice(["fp32", "fp32", "bf16"]), residual=rng.random() < 0.5, **opts)
        else:
            if call == "embedding_grad":
                opts["tied"] = rng.random() < 0.3
            c = _embed(call, _log_uniform(rng, 1, 131072), _log_uniform(rng, 100, 160000), _width(rng, 32, 8192),
                       table=rng.choice(["fp32", "fp32", "bf16", "fp16"]), masked=rng.choice([0.0, 0.1, 0.5]), **opts)
        if work(c)["bytes"] <= most:
            return c


# ------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 41)
    return g


def _matrix(case, rows, cols, dtype):
    """A matrix with the case's padding after each row and its start moved."""
    flat = torch.zeros(rows * (cols + case["pad"]) + 8, dtype=TYPES[dtype], device="cuda")
    return flat[case["shift"]:case["shift"] + rows * (cols + case["pad"])].view(rows, cols + case["pad"])[:, :cols]


def _filled(case, values, dtype):
    return _matrix(case, values.shape[0], values.shape[1], dtype).copy_(values)


def _moments(h, kind):
    """Mean and 1 / sqrt(variance + eps) of the rows as the forward pass hands them on, a few rows at a time."""
    mean, rstd = [], []
    for part in h.split(max(1, (1 << 25) // h.shape[1])):
        x = part.double()
        mu = x.mean(1) if kind == "layer" else torch.zeros(x.shape[0], dtype=torch.float64, device=x.device)
        mean.append(mu)
        rstd.append(((x - mu[:, None]).square().mean(1) + EPS[kind]).rsqrt())
    return torch.cat(mean).float(), torch.cat(rstd).float()


def _norm_inputs(case, seed):
    g, n, d, dtype = _generator(seed), case["rows"], case["cols"], case["dtype"]

    def randn(*size):
        return torch.randn(*size, generator=g, device="cuda")

    s = {}
    # channels of unequal size, a few of them large, about means of their own; tokens of unequal size
    channel = torch.exp(0.4 * randn(d))
    channel = torch.where(torch.rand(d, generator=g, device="cuda") < 0.004, 20.0 * channel, channel)
    stream = (randn(n, d).mul_(channel).add_(0.3 * randn(d))).mul_(torch.exp(0.5 * randn(n, 1)))
    s["weight"] = (1.0 + 0.2 * randn(d)).to(TYPES[case["weight"]])
    if case["call"] == "norm":
        if case["residual"]:
            s["residual"] = _filled(case, stream, dtype)
            s["x"] = _filled(case, randn(n, d).mul_(0.3), dtype)
        else:
            s["residual"], s["x"] = None, _filled(case, stream, dtype)
        s["bias"] = (0.1 * randn(d)).to(TYPES[case["weight"]]) if case["kind"] == "layer" else None
        return s
    s["h"] = _filled(case, stream, dtype)
    del stream
    s["mean"], s["rstd"] = _moments(s["h"], case["kind"])
    size = (64.0 if dtype == "fp16" else 1.0) * 0.01
    s["dy"] = _filled(case, randn(n, d).mul_(torch.exp(randn(n, 1))).mul_(size), dtype)
    s["dh"] = _filled(case, randn(n, d).mul_(size), dtype) if case["residual"] else None
    return s


def _embed_inputs(case, seed):
    g, n, v, d = _generator(seed), case["tokens"], case["vocab"], case["cols"]
    # frequencies as in text: the k-th commonest token about 1 / (k + 10) as often
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    rank = (10.0 * ((v + 10.0) / 10.0) ** u - 10.0).long().clamp(0, v - 1)
    tokens = torch.randperm(v, generator=g, device="cuda")[rank]
    padding = torch.rand(n, generator=g, device="cuda") < case["masked"]
    s = {"tokens": torch.where(padding, torch.full_like(tokens, -100), tokens)}
    if case["call"] == "embedding":
        s["table"] = (0.02 * torch.randn(v, d, generator=g, device="cuda")).to(TYPES[case["table"]])
        s["scale"] = math.sqrt(d)
        return s
    size = 0.64 if case["dtype"] == "fp16" else 0.01
    s["grad"] = _filled(case, torch.randn(n, d, generator=g, device="cuda").mul_(size), case["dtype"])
    s["scale"] = 0.5
    if case["tied"]:
        s["out"] = (size * torch.randn(v, d, generator=g, device="cuda")).to(TYPES[case["table"]])
    else:
        s["out"] = torch.zeros(v, d, dtype=TYPES[case["table"]], device="cuda")
    return s


def prepare(case, seed):
    """The inputs, and the buffers that a training loop keeps for the results."""
    if case["call"] in ("norm", "norm_grad"):
        s = dict(_norm_inputs(case, seed), case=case)
        n, d = case["rows"], case["cols"]
        if case["call"] == "norm":
            s["y"] = _matrix(case, n, d, case["dtype"])
            s["h"] = _matrix(case, n, d, case["dtype"]) if case["residual"] else None
        else:
            s["dx"] = _matrix(case, n, d, case["dtype"])
        return s
    s = dict(_embed_inputs(case, seed), case=case)
    if case["call"] == "embedding":
        s["out"] = _matrix(case, case["tokens"], case["cols"], case["dtype"])
    return s


# -------------------------------------------------------------- plain forms
def _plain_norm(s):
    kind, x = s["case"]["kind"], s["x"].float()
    out = {}
    if s["residual"] is not None:
        s["h"].copy_(x + s["residual"].float())
        out["h"] = s["h"]
        x = s["h"].float()
    if kind == "layer":
        mean = x.mean(1, keepdim=True)
        x = x - mean
        out["mean"] = mean[:, 0]
    rstd = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS[kind])
    y = x * rstd * s["weight"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    s["y"].copy_(y)
    out["y"], out["rstd"] = s["y"], rstd[:, 0]
    return out


def _plain_norm_grad(s):
    layer = s["case"]["kind"] == "layer"
    dy, x = s["dy"].float(), s["h"].float()
    if layer:
        x = x - s["mean"][:, None]
    x = x * s["rstd"][:, None]
    a = dy * s["weight"].float()
    dx = a - x * (a * x).mean(1, keepdim=True)
    if layer:
        dx = dx - a.mean(1, keepdim=True)
    dx = dx * s["rstd"][:, None]
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    s["dx"].copy_(dx)
    out = {"dx": s["dx"], "dweight": (dy * x).sum(0).to(s["weight"].dtype)}
    if layer:
        out["dbias"] = dy.sum(0).to(s["weight"].dtype)
    return out


def _plain_embedding(s):
    t = s["tokens"]
    rows = s["table"][t.clamp(min=0)].float() * s["scale"]
    s["out"].copy_(torch.where((t >= 0)[:, None], rows, torch.zeros_like(rows)))
    return {"out": s["out"]}


def _plain_embedding_grad(s):
    t, held = s["tokens"], s["tokens"] >= 0
    total = torch.zeros(s["out"].shape, device="cuda")
    total.index_add_(0, t[held], s["grad"][held].float())
    total = total * s["scale"]
    s["out"].copy_(s["out"].float() + total if s["case"]["tied"] else total)
    return {"out": s["out"]}


# ------------------------------------------------------------ the operators
def _own_run(s):
    from paper_2609_35701_gb300 import meq

    case = s["case"]
    if case["call"] == "norm":
        if case["kind"] == "layer":
            r = meq.layer_norm(s["x"], s["weight"], s["bias"], residual=s["residual"], eps=EPS["layer"], y=s["y"], h=s["h"])
            out = {"y": r.y, "mean": r.mean, "rstd": r.rstd}
        else:
            r = meq.rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS["rms"], y=s["y"], h=s["h"])
            out = {"y": r.y, "rstd": r.rstd}
        if case["residual"]:
            out["h"] = r.h
        return out
    if case["call"] == "norm_grad":
        if case["kind"] == "layer":
            r = meq.layer_norm_grad(s["dy"], s["h"], s["weight"], s["mean"], s["rstd"], dh=s["dh"], dx=s["dx"])
            return {"dx": r.dx, "dweight": r.dweight, "dbias": r.dbias}
        r = meq.rms_norm_grad(s["dy"], s["h"], s["weight"], s["rstd"], dh=s["dh"], dx=s["dx"])
        return {"dx": r.dx, "dweight": r.dweight}
    if case["call"] == "embedding":
        return {"out": meq.embedding(s["tokens"], s["table"], scale=s["scale"], out=s["out"])}
    return {"out": meq.embedding_grad(s["grad"], s["tokens"], s["out"], scale=s["scale"], accumulate=case["tied"])}


def run(state):
    if own:
        return _own_run(state)
    plain = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "embedding": _plain_embedding, "embedding_grad": _plain_embedding_grad}
    return plain[state["case"]["call"]](state)


# --------------------------------------------------------------------- work
def _distinct(n, vocab):
    """Distinct tokens to be expected among n of the distribution above."""
    norm, total, low = math.log((vocab + 10.0) / 10.0), 0.0, 0.0
    while low < vocab:   # ranks in blocks of a constant ratio
        high = min(float(vocab), max(low + 1.0, low * 1.05))
        p = math.log((high + 10.0) / (low + 10.0)) / norm / (high - low)
        total += (high - low) * -math.expm1(n * math.log1p(-min(p, 1.0 - 1e-12)))
        low = high
    return total


def work(case):
    size = float(BYTES[case["dtype"]])
    if case["call"] in ("norm", "norm_grad"):
        numel, vectors = float(case["rows"] * case["cols"]), (2 if case["kind"] == "layer" else 1)
        per_row = 4.0 * vectors * case["rows"]
        if case["call"] == "norm":
            return {"bytes": (4 if case["residual"] else 2) * size * numel + per_row + vectors * case["cols"] * BYTES[case["weight"]],
                    "flops": 8.0 * numel}
        return {"bytes": (4 if case["residual"] else 3) * size * numel + per_row + (vectors + 1) * case["cols"] * BYTES[case["weight"]],
                "flops": 14.0 * numel}
    n, d = float(case["tokens"]), case["cols"]
    held = max(1.0, n * (1.0 - case["masked"]))
    rows = _distinct(held, case["vocab"])
    if case["call"] == "embedding":
        return {"bytes": 8.0 * n + rows * d * BYTES[case["table"]] + n * d * size, "flops": held * d}
    written = 2.0 * rows if case["tied"] else float(case["vocab"])
    return {"bytes": 8.0 * n + held * d * size + written * d * BYTES[case["table"]], "flops": 2.0 * held * d}


# -------------------------------------------------------------------- 64 bits
def _exact_norm(case, seed):
    s, kind = _norm_inputs(case, seed), case["kind"]
    n, d = s["x"].shape
    out = {k: torch.empty(n, d, dtype=torch.float64, device="cuda") for k in (["y", "h"] if case["residual"] else ["y"])}
    w = s["weight"].double()
    mean, rstd = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.empty(n, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 25) // d)
    for i in range(0, n, step):
        x = s["x"][i:i + step].double()
        if case["residual"]:
            x = (x + s["residual"][i:i + step].double()).to(TYPES[case["dtype"]]).double()   # the stream as it is held
            out["h"][i:i + step] = x
        var = x.square().mean(1)
        if kind == "layer":
            var, mu = torch.var_mean(x, 1, correction=0)
            mean[i:i + step] = mu
        rstd[i:i + step] = (var + EPS[kind]) ** -0.5
        y = (x - mean[i:i + step, None]) * (rstd[i:i + step, None] * w)
        out["y"][i:i + step] = y + s["bias"].double() if s["bias"] is not None else y
    out["rstd"] = rstd
    if kind == "layer":
        out["mean"] = mean
    return out


def _exact_norm_grad(case, seed):
    s, layer = _norm_inputs(case, seed), case["kind"] == "layer"
    n, d = s["dy"].shape
    w = s["weight"].double()
    out = {"dx": torch.empty(n, d, dtype=torch.float64, device="cuda"), "dweight": torch.zeros_like(w)}
    if layer:
        out["dbias"] = torch.zeros_like(w)
    step = max(1, (1 << 25) // d)
    for i in range(0, n, step):
        at = slice(i, i + step)
        r = s["rstd"][at, None].double()
        xhat = (s["h"][at].double() - s["mean"][at, None].double()) * r if layer else s["h"][at].double() * r
        dy = s["dy"][at].double()
        a = dy * w
        inner = (torch.einsum("ij,ij->i", a, xhat) / d)[:, None] * xhat + (a.mean(1, keepdim=True) if layer else 0.0)
        dx = r * (a - inner)
        out["dx"][at] = dx + s["dh"][at].double() if s["dh"] is not None else dx
        out["dweight"] += torch.einsum("ij,ij->j", dy, xhat)
        if layer:
            out["dbias"] += dy.sum(0)
    return out


def _exact_embedding(case, seed):
    s = _embed_inputs(case, seed)
    out = torch.zeros(case["tokens"], case["cols"], dtype=torch.float64, device="cuda")
    held = torch.nonzero(s["tokens"] >= 0)[:, 0]
    out[held] = s["table"][s["tokens"][held]].double() * s["scale"]
    return {"out": out}


def _exact_embedding_grad(case, seed):
    s = _embed_inputs(case, seed)
    t = s["tokens"]
    order = torch.argsort(t, stable=True)
    order = order[t[order] >= 0]
    tokens, counts = torch.unique_consecutive(t[order], return_counts=True)
    out = s["out"].double() if case["tied"] else torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    if tokens.numel():
        sums = torch.segment_reduce(s["grad"][order].double(), "sum", lengths=counts, axis=0)
        out[tokens] += s["scale"] * sums
    return {"out": out}


def exact(case, seed):
    call = {"norm": _exact_norm, "norm_grad": _exact_norm_grad, "embedding": _exact_embedding, "embedding_grad": _exact_embedding_grad}
    return call[case["call"]](case, seed)
