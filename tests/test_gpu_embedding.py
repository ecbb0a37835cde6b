"""The embedding and the gradient of its table against plain 64-bit arithmetic.

Tolerances, u = 2^-24. A looked-up value is one product, rounded to fp32 and to its type. Of a row of the gradient
that c tokens share, a term is added at most K = min(c, 48 + c / 32) times (32 in a chunk, c / 32 chunks of at
least 4 in one of 8 warps, 8 warps), and the sum is scaled, and where it accumulates added, in one rounding:
  T = (K + 1) u |scale| sum|g| + u |result|, and half a step of the type.
"""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF_ULP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
LEAST = {"fp32": 1e-37, "bf16": 1e-37, "fp16": 2.0 ** -25}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def meq():
    import __graft_entry__

    __graft_entry__.build()
    from paper_2609_35701_gb300 import meq as m

    return m


def _matrix(rows, cols, dtype, pad=0, shift=0, seed=None, fill=0.0):
    flat = torch.full((rows * (cols + pad) + shift,), fill, dtype=DT[dtype], device="cuda")
    m = flat[shift:].view(rows, cols + pad)[:, :cols]
    if seed is not None:
        m.copy_(torch.randn(rows, cols, generator=torch.Generator().manual_seed(seed)))
    return m


def _tokens(n, vocab, how, seed=0):
    g = torch.Generator().manual_seed(seed)
    if how == "uniform":
        t = torch.randint(0, vocab, (n,), generator=g)
    elif how == "skewed":
        t = (vocab ** torch.rand(n, generator=g, dtype=torch.float64)).long().clamp(max=vocab) - 1
    elif how == "one":
        t = torch.full((n,), vocab - 1)
    elif how == "distinct":
        t = torch.randperm(vocab, generator=g)[:n]
    elif how == "two":   # runs that end inside chunks
        t = (torch.arange(n) >= n // 3).long() * (vocab - 1)
    else:
        t = torch.full((n,), -1)
    if how in ("uniform", "skewed"):
        t[torch.rand(n, generator=g) < 0.1] = -100
    return t.cuda()


def _round(want, tol, dtype):
    return tol + HALF_ULP[dtype] * (want.abs() + tol) + LEAST[dtype]


def _check_grad(got, grad, tokens, scale, before, dtype):
    """got against the sums in 64 bits on the device (index_add_ in doubles), every row of them."""
    vocab, scale = got.shape[0], float(np.float32(scale))
    held = (tokens >= 0) & (tokens < vocab)
    t, g = tokens[held], grad[held].double()
    sums = torch.zeros(got.shape, dtype=torch.float64, device="cuda").index_add_(0, t, g)
    sizes = torch.zeros(got.shape, dtype=torch.float64, device="cuda").index_add_(0, t, g.abs())
    count = torch.bincount(t, minlength=vocab).double()[:, None]
    want = scale * sums + (before.double() if before is not None else 0.0)
    deep = torch.minimum(count, 48 + count / 32) + 1
    tol = _round(want, deep * U * abs(scale) * sizes + U * want.abs(), dtype)
    untouched = count[:, 0] == 0
    if before is not None:
        assert torch.equal(got[untouched], before[untouched])
    else:
        assert not got[untouched].any()
    bad = ~((got.double() - want).abs() <= tol)
    assert not bool(bad.any()), (torch.nonzero(bad)[:5].tolist(), got[bad][:5].tolist(), want[bad][:5].tolist())


# tokens, vocab, cols, pad, shift
LOOKUPS = [(1, 1, 1, 0, 0), (3, 5, 8, 0, 0), (16, 1000, 768, 0, 0), (33, 70, 7, 0, 1), (200, 321, 96, 8, 0), (100, 50, 1025, 0, 0), (77, 500, 100, 0, 4),
           (5, 9, 5461, 3, 0), (400, 1000, 2048, 0, 8), (3000, 40000, 64, 0, 0)]


@pytest.mark.parametrize("table_type", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n,vocab,cols,pad,shift", LOOKUPS)
def test_lookup(meq, table_type, dtype, n, vocab, cols, pad, shift):
    table, tokens, scale = _matrix(vocab, cols, table_type, pad, shift, seed=1), _tokens(n, vocab, "uniform", 2), 11.3
    out = meq.embedding(tokens, table, scale=scale, dtype=DT[dtype])
    assert out.shape == (n, cols) and out.dtype is DT[dtype]
    want = table.double()[tokens.clamp(min=0)] * float(np.float32(scale))
    want[tokens < 0] = 0.0
    assert bool(((out.double() - want).abs() <= _round(want, U * want.abs(), dtype)).all())
    given = _matrix(n, cols, dtype, pad=5, shift=1, fill=7.0)
    version = given._version
    assert meq.embedding(tokens, table, scale=scale, out=given) is given and torch.equal(given, out) and given._version > version
    if cols > 1:
        assert bool((given.as_strided((n - 1, 5), (cols + 5, 1), given.storage_offset() + cols) == 7.0).all())


def test_lookup_of_no_token(meq):
    table = _matrix(10, 24, "bf16", seed=1)
    t = torch.tensor([3, -1, 9, 10, 1 << 40, -(1 << 40)], device="cuda")
    for x in (table, _matrix(10, 25, "bf16", seed=1)):
        out = meq.embedding(t, x)
        assert torch.equal(out[0], x[3]) and torch.equal(out[2], x[9]) and not out[1].any() and not out[5].any()
        assert bool(out[3].isnan().all()) and bool(out[4].isnan().all())
        assert meq.embedding(t[:0], x).shape == (0, x.shape[1])


# tokens, vocab, cols, pad, shift
GRADS = [(1, 1, 1, 0, 0), (1, 1000, 768, 0, 0), (2, 3, 8, 0, 0), (24, 32000, 96, 0, 0), (31, 40, 7, 0, 1), (33, 511, 64, 8, 0), (100, 512, 100, 0, 0),
         (257, 513, 1025, 0, 0), (1000, 30, 256, 0, 8), (1000, 50001, 33, 1, 3), (3000, 1000, 768, 0, 0), (5000, 70, 512, 0, 0), (5000, 300001, 24, 0, 0),
         (9000, 2000, 2048, 0, 0), (40000, 10000, 40, 0, 0), (70001, 3000, 136, 0, 0),
         (128, 90, 24, 0, 0), (129, 90, 24, 0, 0), (255, 400, 1032, 0, 0), (256, 60, 24, 0, 0), (257, 400, 24, 0, 0), (16384, 700, 16, 0, 0), (16385, 700, 16, 0, 0), (200001, 5000, 8, 0, 0)]


@pytest.mark.parametrize("out_type", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n,vocab,cols,pad,shift", GRADS)
def test_gradient(meq, out_type, dtype, n, vocab, cols, pad, shift):
    how = "uniform" if n % 2 else "skewed"
    grad, tokens, scale = _matrix(n, cols, dtype, pad, shift, seed=n), _tokens(n, vocab, how, cols), 0.37
    out = _matrix(vocab, cols, out_type, fill=7.0)
    version = out._version
    assert meq.embedding_grad(grad, tokens, out, scale=scale) is out and out._version > version
    _check_grad(out, grad, tokens, scale, None, out_type)
    padded = _matrix(vocab, cols, out_type, pad=5, shift=1, fill=7.0)
    meq.embedding_grad(grad, tokens, padded, scale=scale)
    assert torch.equal(padded, out)
    if vocab > 1:
        assert bool((padded.as_strided((vocab - 1, 5), (cols + 5, 1), padded.storage_offset() + cols) == 7.0).all())
    before = _matrix(vocab, cols, out_type, pad=3, shift=1, seed=5)
    got = _matrix(vocab, cols, out_type, pad=3, shift=1, fill=7.0)
    got.copy_(before)
    meq.embedding_grad(grad, tokens, got, scale=scale, accumulate=True)
    _check_grad(got, grad, tokens, scale, before, out_type)
    if vocab > 1:
        assert bool((got.as_strided((vocab - 1, 3), (cols + 3, 1), got.storage_offset() + cols) == 7.0).all())


@pytest.mark.parametrize("how", ["one", "distinct", "two", "none"])
@pytest.mark.parametrize("n,cols", [(5, 16), (128, 96), (256, 40), (250, 33), (257, 40), (1000, 1025), (4096, 264), (30000, 64), (100000, 8)])
def test_gradient_of_runs(meq, how, n, cols):
    """One token everywhere, each once, two long runs, none at all."""
    vocab = max(n, 700)
    grad, tokens = _matrix(n, cols, "bf16", seed=n), _tokens(n, vocab, how, 1)
    out = _matrix(vocab, cols, "fp32", fill=7.0)
    meq.embedding_grad(grad, tokens, out)
    _check_grad(out, grad, tokens, 1.0, None, "fp32")


def test_gradient_over_a_vast_vocabulary(meq):
    """More rows than a block's marks cover at a time, and four digits to sort by."""
    vocab, n = 160000000, 3000
    tokens = torch.randint(0, vocab, (n,), generator=torch.Generator().manual_seed(1)).cuda()
    tokens[:4] = torch.tensor([0, vocab - 1, 524288, 524287])
    grad = torch.ones(n, 1, dtype=torch.bfloat16, device="cuda")
    out = torch.full((vocab, 1), 7.0, dtype=torch.bfloat16, device="cuda")
    meq.embedding_grad(grad, tokens, out)
    want, counts = torch.unique(tokens, return_counts=True)
    at = torch.nonzero(out[:, 0])[:, 0]
    assert torch.equal(at, want) and torch.equal(out[at, 0].long(), counts)


def test_rows_that_a_32_bit_offset_does_not_reach(meq):
    n, cols = 300001, 8200                       # 2.46e9 elements of gradient
    tokens = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    tokens[-3:] = torch.tensor([5, 2, 5])
    grad = torch.empty(n, cols, dtype=torch.bfloat16, device="cuda")
    grad[-3:] = _matrix(3, cols, "bf16", seed=1)
    out = _matrix(7, cols, "fp32", fill=7.0)
    meq.embedding_grad(grad, tokens, out)
    _check_grad(out, grad[-3:], tokens[-3:], 1.0, None, "fp32")
    table = grad                                  # as a table: its last rows
    t = torch.tensor([n - 1, n - 3], device="cuda")
    assert torch.equal(meq.embedding(t, table), table[t])


def test_nonfinite_gradients_stay_in_their_rows(meq):
    tokens = torch.tensor([4, 2, 4, 6, -1, 99], device="cuda")
    for cols in (16, 17):
        grad = _matrix(6, cols, "bf16", seed=1)
        grad[1] = float("nan")
        grad[3, 5] = float("inf")
        grad[4:] = float("nan")                   # of a padding token, and of one beyond the table
        out = meq.embedding_grad(grad, tokens, torch.empty(8, cols, device="cuda"))
        assert bool(out[2].isnan().all()) and bool(out[6, 5].isinf()) and int(out[6].isfinite().sum()) == cols - 1
        assert bool(out[[0, 1, 3, 4, 5, 7]].isfinite().all()) and bool(out[4].any())


@pytest.mark.parametrize("n,vocab,cols", [(1, 3000, 64), (700, 3000, 768), (20000, 900, 264), (3000, 5000, 1025)])
def test_results_repeat_and_calls_overlap(meq, n, vocab, cols):
    """The same bits again, from several streams at once, and from captured graphs on new inputs."""
    grads, tokens = [_matrix(n, cols, "bf16", seed=s) for s in (1, 2)], [_tokens(n, vocab, "skewed", s) for s in (3, 4)]
    want = [meq.embedding_grad(g, t, torch.empty(vocab, cols, device="cuda")) for g, t in zip(grads, tokens)]
    looked = [meq.embedding(t, w, dtype=torch.bfloat16) for t, w in zip(tokens, want)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty(vocab, cols, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for g, t, o, s in zip(grads, tokens, outs, streams):
            meq.embedding_grad(g, t, o, stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
    g, t = grads[0].clone(), tokens[0].clone()
    graphs, results = [], []
    for s, o in zip(streams, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            meq.embedding_grad(g, t, o)
            results.append(meq.embedding(t, o, dtype=torch.bfloat16))
        graphs.append(graph)
    for i in (1, 0):
        g.copy_(grads[i])
        t.copy_(tokens[i])
        for graph, o, r in zip(graphs, outs, results):
            graph.replay()
            assert torch.equal(o, want[i]) and torch.equal(r, looked[i])


CAPTURED_FIRST = """
import sys, torch
sys.path.insert(0, {root!r})
from paper_2609_35701_gb300 import meq
t = torch.randint(0, 500, (3000,), device="cuda")
table, w = torch.randn(500, 96, device="cuda"), torch.ones(96, device="cuda")
out = torch.empty_like(table)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    x = meq.embedding(t, table)
    r = meq.layer_norm(x, w)
    g = meq.layer_norm_grad(r.y, x, w, r.mean, r.rstd)
    meq.embedding_grad(g.dx, t, out)
graph.replay()
torch.cuda.synchronize()
held = out.clone()
x = meq.embedding(t, table)
r = meq.layer_norm(x, w)
meq.embedding_grad(meq.layer_norm_grad(r.y, x, w, r.mean, r.rstd).dx, t, out)
assert torch.equal(held, out) and bool(out.any())
"""


def test_a_process_may_begin_with_a_capture(meq):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", CAPTURED_FIRST.format(root=root)], capture_output=True, text=True, timeout=120)
    assert done.returncode == 0, done.stderr[-2000:]


def test_gradient_is_the_lookups_transpose(meq):
    """<embedding(E + d U) - embedding(E - d U), g> / 2d = <U, dE>: the lookup is linear, so any d will do."""
    n, vocab, cols, scale = 300, 90, 40, 0.75
    tokens = _tokens(n, vocab, "skewed", 1)
    table, u, grad = (_matrix(r, cols, "fp32", seed=s) for r, s in ((vocab, 2), (vocab, 3), (n, 4)))
    up, down = (meq.embedding(tokens, table + d * u, scale=scale).double() for d in (1.0, -1.0))
    got = float((meq.embedding_grad(grad, tokens, torch.empty_like(table), scale=scale).double() * u.double()).sum())
    want = float(((up - down) / 2 * grad.double()).sum())
    # a sum, a product and a difference in fp32 on either side, and the additions of a row
    size = float(((up.abs() + down.abs()) * grad.double().abs()).sum()) + float((u.abs().double() * 300).sum())
    assert abs(got - want) <= 100 * U * size


def test_refusals(meq):
    t, e, g = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(10, 8, device="cuda"), torch.zeros(4, 8, device="cuda")
    bad = [lambda: meq.embedding(t.int(), e), lambda: meq.embedding(t.cpu(), e), lambda: meq.embedding(t, e.cpu()), lambda: meq.embedding(t, e.double()),
           lambda: meq.embedding(t, e[0]), lambda: meq.embedding(t, e.T), lambda: meq.embedding(t, e, out=g[:3]), lambda: meq.embedding(t, e, out=g[:, :4]),
           lambda: meq.embedding(t, e, out=g, dtype=torch.float16), lambda: meq.embedding(t, e, dtype=torch.float64),
           lambda: meq.embedding(torch.zeros(8, dtype=torch.int64, device="cuda")[::2], e), lambda: meq.embedding(t, e, out=g[:1].expand(4, 8)),
           lambda: meq.embedding_grad(g, t[:3], e), lambda: meq.embedding_grad(g, t, e[:, :4]), lambda: meq.embedding_grad(g.double(), t, e),
           lambda: meq.embedding_grad(g, t, e.cpu()), lambda: meq.embedding_grad(g.cpu(), t, e), lambda: meq.embedding_grad(g, t, e[:1].expand(10, 8))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(i)


def test_results_that_a_32_bit_offset_does_not_reach(meq):
    """Rows of the result 1.2e9 elements apart, of the lookup and of the table's gradient, written and added to."""
    apart = 1200000000
    far = torch.empty(2 * apart + 2000, dtype=torch.bfloat16, device="cuda")
    for n, cols in ((5, 96), (300, 1025)):
        tokens = torch.arange(n, device="cuda") % 4                # 3 is padding
        tokens[tokens == 3] = -1
        grad = _matrix(n, cols, "bf16", seed=1)
        out = far.as_strided((3, cols), (apart, 1))
        before = _matrix(3, cols, "bf16", seed=2)
        for held in (None, before):
            if held is not None:
                out.copy_(held)
            meq.embedding_grad(grad, tokens, out, accumulate=held is not None)
            _check_grad(out, grad, tokens, 1.0, held, "bf16")
        table = _matrix(4, cols, "bf16", seed=3)
        t = torch.tensor([3, 0, 2], device="cuda")
        assert torch.equal(meq.embedding(t, table, out=out), table[t])


def test_one_token_in_up_to_256(meq):
    """One warp adds up its rows in turn: each is added at most n times."""
    for n in (97, 256):
        grad, tokens = _matrix(n, 264, "fp32", seed=n), torch.full((n,), 5, device="cuda")
        out = meq.embedding_grad(grad, tokens, torch.empty(9, 264, device="cuda"))
        sizes, want = grad.double().abs().sum(0), grad.double().sum(0)
        assert bool(((out[5].double() - want).abs() <= (n + 1) * U * sizes + U * want.abs()).all())
        assert not out[[0, 1, 2, 3, 4, 6, 7, 8]].any()
