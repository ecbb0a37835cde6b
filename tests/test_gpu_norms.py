"""Layer norm, RMS norm and their backward pass against plain 64-bit arithmetic.

Tolerances, u = 2^-24. A row's sum adds a term at most D = 64 + cols / 512 times (32 in a thread or cols / 512
of them where rows are read again, and the trees), so
  T(mu) = (D + 1) u mean|h|
  rel(var) = (D + 4) u + T(mu)^2 / var, and half of it, times var / (var + eps), with 3 u for the root: rel(rstd)
  T(y) = |w| rstd (T(mu) + 2 u |h - mu|) + |y - b| (rel(rstd) + 3 u) + 2 u |y|.
Backward, mu and rstd given: xhat is off by 3 u |xhat|, so
  T(c1) = (D + 6) u mean|a xhat|, T(c2) = (D + 3) u mean|a|
  T(dx) = rstd (4 u (|a| + |c2| + 2 |xhat c1|) + T(c2) + |xhat| T(c1)) + 2 u (|dx| + |dh|)
and sums over rows add a term at most R = 96 + rows / 100 times (rows / 150 in a thread, the rest in trees):
  T(dw) = (R + 5) u sum|dy xhat|, T(db) = (R + 1) u sum|dy|.
Each with half a step of its type on top.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF_ULP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
LEAST = {"fp32": 1e-37, "bf16": 1e-37, "fp16": 2.0 ** -25}
U = 2.0 ** -24
EPS = 1e-5
EPS32 = float(np.float32(EPS))
EPS_RMS = float(np.float32(1e-6))  # rms_norm's own


@pytest.fixture(scope="module")
def meq():
    import __graft_entry__

    __graft_entry__.build()
    from paper_2609_35701_gb300 import meq as m

    return m


def _np(t):
    return t.detach().cpu().double().numpy()


def _matrix(rows, cols, dtype, pad=0, shift=0, fill=0.0):
    flat = torch.full((rows * (cols + pad) + shift,), fill, dtype=DT[dtype], device="cuda")
    return flat[shift:].view(rows, cols + pad)[:, :cols]


def _random(rows, cols, dtype, seed, pad=0, shift=0, spread=1.0, offset=0.0):
    g = torch.Generator().manual_seed(seed)
    x = spread * torch.randn(rows, cols, generator=g) * torch.exp(0.5 * torch.randn(rows, 1, generator=g)) + offset
    return _matrix(rows, cols, dtype, pad, shift).copy_(x)


def _vector(cols, dtype, seed, centre):
    return (centre + 0.3 * torch.randn(cols, generator=torch.Generator().manual_seed(seed))).to(DT[dtype]).cuda()


def _round(want, tol, dtype):
    return tol + HALF_ULP[dtype] * (np.abs(want) + tol) + LEAST[dtype]


def _within(got, want, tol):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], tol[bad][:5] if tol.shape == got.shape else tol)


def _statistics(h, centred, eps=EPS32):
    """mu, rstd and what they may be off by."""
    n = h.shape[1]
    d = 64 + n / 512
    mu = h.mean(1) if centred else np.zeros(len(h))
    tmu = (d + 1) * U * np.abs(h).mean(1) if centred else np.zeros(len(h))
    var = np.square(h - mu[:, None]).mean(1)
    rel = 0.5 * ((d + 4) * U * var + tmu ** 2) / (var + eps) + 3 * U
    return mu, tmu, 1 / np.sqrt(var + eps), rel


def _check_forward(r, h, w, b, centred, dtype, eps=EPS32):
    mu, tmu, rstd, rel = _statistics(h, centred, eps)
    _within(_np(r.rstd), rstd, rstd * rel)
    if centred:
        _within(_np(r.mean), mu, tmu + U * np.abs(mu) + 1e-37)
    d = h - mu[:, None]
    y0 = d * rstd[:, None] * w
    want = y0 + b
    tol = np.abs(w) * rstd[:, None] * (tmu[:, None] + 2 * U * np.abs(d)) + np.abs(y0) * (rel[:, None] + 3 * U) + 2 * U * np.abs(want)
    _within(_np(r.y), want, _round(want, tol, dtype))


def _check_backward(r, dy, h, w, mu, rstd, dh, centred, dtype, weight_type):
    rows, n = dy.shape
    d, deep = 64 + n / 512, 96 + rows / 100
    mu = mu[:, None] if centred else 0.0
    xhat, a = (h - mu) * rstd[:, None], dy * w
    c1, c2 = (a * xhat).mean(1, keepdims=True), a.mean(1, keepdims=True) * (1.0 if centred else 0.0)
    want = rstd[:, None] * (a - c2 - xhat * c1) + dh
    tc1, tc2 = (d + 6) * U * np.abs(a * xhat).mean(1, keepdims=True), (d + 3) * U * np.abs(a).mean(1, keepdims=True) * centred
    tol = rstd[:, None] * (4 * U * (np.abs(a) + np.abs(c2) + 2 * np.abs(xhat * c1)) + tc2 + np.abs(xhat) * tc1)
    tol = tol + 2 * U * (np.abs(want) + np.abs(dh))
    _within(_np(r.dx), want, _round(want, tol, dtype))
    if r.dweight is not None:
        want = (dy * xhat).sum(0)
        _within(_np(r.dweight).reshape(-1), want, _round(want, (deep + 5) * U * np.abs(dy * xhat).sum(0), weight_type))
    if centred and r.dbias is not None:
        want = dy.sum(0)
        _within(_np(r.dbias).reshape(-1), want, _round(want, (deep + 1) * U * np.abs(dy).sum(0), weight_type))


def _forward(meq, kind, x, w, b, **kw):
    return meq.layer_norm(x, w, b, eps=EPS, **kw) if kind == "layer" else meq.rms_norm(x, w, eps=EPS, **kw)


def _backward(meq, kind, dy, h, w, r, **kw):
    return meq.layer_norm_grad(dy, h, w, r.mean, r.rstd, **kw) if kind == "layer" else meq.rms_norm_grad(dy, h, w, r.rstd, **kw)


# rows, cols, pad, shift
SIZES = [(3, 1, 0, 0), (5, 2, 1, 1), (4, 7, 0, 0), (9, 8, 0, 3), (70, 31, 0, 0), (33, 32, 8, 0), (200, 64, 0, 0), (37, 100, 0, 2),
         (1, 128, 0, 0), (65, 128, 64, 0), (16, 255, 1, 1), (19, 256, 0, 0), (17, 264, 0, 8), (500, 768, 0, 0), (3, 1000, 0, 1), (700, 1024, 0, 0),
         (163, 1025, 0, 0), (6, 1032, 0, 0), (30, 2048, 8, 0), (5, 2055, 2, 5), (160, 4096, 0, 0), (7, 4097, 0, 0), (9, 5461, 0, 0), (12, 6000, 0, 0),
         (5, 8192, 64, 8), (4, 11008, 0, 0), (3, 12289, 0, 1), (4, 16384, 0, 0), (2, 16391, 0, 0), (3, 20480, 0, 0), (2, 70001, 0, 0)]


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,cols,pad,shift", SIZES)
def test_forward_and_backward(meq, kind, dtype, rows, cols, pad, shift):
    weight_type = {"fp32": "fp32", "bf16": "fp32", "fp16": "bf16"}[dtype] if cols % 2 else dtype
    x, w, b = _random(rows, cols, dtype, cols, pad, shift, offset=0.5), _vector(cols, weight_type, 1, 1.0), _vector(cols, weight_type, 2, 0.0)
    r = _forward(meq, kind, x, w, b if kind == "layer" else None)
    assert r.h is x
    _check_forward(r, _np(x), _np(w), _np(b) if kind == "layer" else 0.0, kind == "layer", dtype)
    dy = _random(rows, cols, dtype, cols + 1, pad, shift)
    g = _backward(meq, kind, dy, x, w, r)
    assert g.dweight.dtype is w.dtype
    _check_backward(g, _np(dy), _np(x), _np(w), _np(r.mean) if kind == "layer" else None, _np(r.rstd), 0.0, kind == "layer", dtype, weight_type)


RESIDUAL = [(5, 24, 0, 0), (40, 100, 3, 1), (300, 768, 0, 0), (21, 1025, 0, 0), (64, 4096, 0, 0), (6, 12000, 1, 0), (3, 20001, 0, 0)]


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,cols,pad,shift", RESIDUAL)
def test_residual_stream(meq, kind, dtype, rows, cols, pad, shift):
    """The stream is written, and normalised as it is held; its own gradient joins the input's."""
    x, res = _random(rows, cols, dtype, 1, 0, 0), _random(rows, cols, dtype, 2, pad, shift, spread=3.0)
    w, b = _vector(cols, "fp32", 3, 1.0), _vector(cols, "fp32", 4, 0.0)
    r = _forward(meq, kind, x, w, b if kind == "layer" else None, residual=res)
    total = _np(x) + _np(res)
    _within(_np(r.h), total, _round(total, U * np.abs(total), dtype))
    _check_forward(r, _np(r.h), _np(w), _np(b) if kind == "layer" else 0.0, kind == "layer", dtype)
    dy, dh = _random(rows, cols, dtype, 5, pad, shift), _random(rows, cols, dtype, 6)
    g = _backward(meq, kind, dy, r.h, w, r, dh=dh)
    _check_backward(g, _np(dy), _np(r.h), _np(w), _np(r.mean) if kind == "layer" else None, _np(r.rstd), _np(dh), kind == "layer", dtype, "fp32")


@pytest.mark.parametrize("rows,cols", [(20000, 96), (5000, 1024), (3000, 4096), (3000, 1031), (800, 17000)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_many_rows(meq, rows, cols, dtype):
    x, dy = _random(rows, cols, dtype, 7, offset=-1.0), _random(rows, cols, dtype, 8)
    w, b = _vector(cols, "fp32", 9, 1.0), _vector(cols, "fp32", 10, 0.0)
    r = meq.layer_norm(x, w, b, eps=EPS)
    _check_forward(r, _np(x), _np(w), _np(b), True, dtype)
    _check_backward(meq.layer_norm_grad(dy, x, w, r.mean, r.rstd), _np(dy), _np(x), _np(w), _np(r.mean), _np(r.rstd), 0.0, True, dtype, "fp32")


WIDTHS = [40, 96, 768, 1025, 4096, 17000]


@pytest.mark.parametrize("cols", WIDTHS)
def test_in_place(meq, cols):
    """y over x, h over the residual, dx over dy, h or dh: the same bits as out of place."""
    rows, w, b = 37, _vector(cols, "fp32", 1, 1.0), _vector(cols, "fp32", 2, 0.0)
    x, res = _random(rows, cols, "bf16", 3), _random(rows, cols, "bf16", 4)
    want = meq.layer_norm(x, w, b, residual=res)
    for swap in (False, True):
        a, c = x.clone(), res.clone()
        versions = a._version, c._version
        got = meq.layer_norm(a, w, b, residual=c, y=c if swap else a, h=a if swap else c)
        assert torch.equal(got.y, want.y) and torch.equal(got.h, want.h) and torch.equal(got.rstd, want.rstd)
        assert got.y is (c if swap else a) and a._version > versions[0] and c._version > versions[1]
    a = x.clone()
    assert torch.equal(meq.rms_norm(a, w, y=a).y, meq.rms_norm(x, w).y)
    dy, dh = _random(rows, cols, "bf16", 5), _random(rows, cols, "bf16", 6)
    g = meq.layer_norm_grad(dy, want.h, w, want.mean, want.rstd, dh=dh)
    for which in range(3):
        t = [dy.clone(), want.h.clone(), dh.clone()]
        got = meq.layer_norm_grad(t[0], t[1], w, want.mean, want.rstd, dh=t[2], dx=t[which])
        assert got.dx is t[which] and torch.equal(got.dx, g.dx) and torch.equal(got.dweight, g.dweight) and torch.equal(got.dbias, g.dbias)


@pytest.mark.parametrize("cols", WIDTHS)
def test_padding_is_left(meq, cols):
    """Nothing but the rows' own elements is written, at either end."""
    rows, w = 11, _vector(cols, "fp32", 1, 1.0)
    x, res, dy = (_random(rows, cols, "bf16", s) for s in (2, 3, 4))
    for pad, shift in ((0, 1), (3, 5), (8, 8)):
        flats = [torch.full((rows * (cols + pad) + shift + 9,), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
        y, h, dx = (f[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] for f in flats)
        r = meq.rms_norm(x, w, residual=res, y=y, h=h)
        g = meq.rms_norm_grad(dy, h, w, r.rstd, dx=dx)
        # rows that start elsewhere in their 16 bytes are added up in another order: each is held against 64 bits
        assert torch.equal(r.h, meq.rms_norm(x, w, residual=res).h)
        _check_forward(r, _np(h), _np(w), 0.0, False, "bf16", EPS_RMS)
        _check_backward(g, _np(dy), _np(h), _np(w), None, _np(r.rstd), 0.0, False, "bf16", "fp32")
        for f, t in zip(flats, (y, h, dx)):
            t.fill_(7.0)
            assert bool((f == 7.0).all())


@pytest.mark.parametrize("cols", WIDTHS)
def test_unusual_rows(meq, cols):
    """Constant rows, a large mean, rows with a NaN, an infinity or an overflowing sum: each alone."""
    x = _random(9, cols, "fp32", 1)
    x[1] = 0.0
    x[2] = 3.0
    x[3] += 1000.0
    x[4, cols // 2] = float("nan")
    x[5, 0] = float("inf")
    x[6, cols - 1] = -float("inf")
    x[7] = 1e25
    x[7, ::2] = -1e25
    w, b = _vector(cols, "fp32", 2, 1.0), _vector(cols, "fp32", 3, 0.0)
    whole = [0, 1, 2, 3, 8]
    r = meq.layer_norm(x, w, b, eps=EPS)
    _check_forward(meq.LayerNorm(r.y[whole], None, r.mean[whole], r.rstd[whole]), _np(x[whole]), _np(w), _np(b), True, "fp32")
    q = meq.rms_norm(x, w, eps=EPS)
    _check_forward(meq.RmsNorm(q.y[whole], None, q.rstd[whole]), _np(x[whole]), _np(w), 0.0, False, "fp32")
    for i in (4, 5, 6, 7):
        assert bool(r.y[i].isnan().all()), i
        assert bool(q.rstd[i].isnan()) and bool(q.y[i].isnan().all()), i
    dy = _random(9, cols, "fp32", 4)
    g = meq.layer_norm_grad(dy, x, w, r.mean, r.rstd)
    for i in (4, 5, 6, 7):
        assert bool(g.dx[i].isnan().all())
    assert bool(g.dx[whole].isfinite().all()) and bool(g.dweight.isnan().all()) and bool(g.dbias.isfinite().all())


def test_constant_rows_and_a_tiny_eps(meq):
    """rstd up to 1e22: its square overflows, the gradient of a constant row, which is rstd (a - mean a), need not."""
    for cols in (96, 1025, 17000):
        x, dy, w = torch.full((4, cols), 2.0, device="cuda"), _random(4, cols, "fp32", 1), torch.ones(cols, device="cuda")
        x[1] = 0.0
        r = meq.layer_norm(x, w, eps=1e-44)
        assert bool((r.y[1] == 0).all()) and bool(r.rstd[1].isfinite())
        g = meq.layer_norm_grad(dy, x, w, r.mean, r.rstd)
        assert bool(g.dx[1].isfinite().all()) and bool(g.dx[1].any())


def test_options(meq):
    """No weight, no bias, given outputs of other types, no rows."""
    for cols in (96, 1025, 17000):
        x, dy = _random(6, cols, "bf16", 1), _random(6, cols, "bf16", 2)
        r = meq.layer_norm(x, eps=EPS)
        _check_forward(r, _np(x), np.ones(cols), 0.0, True, "bf16")
        b = _vector(cols, "fp16", 3, 0.0)
        _check_forward(meq.layer_norm(x, None, b, eps=EPS), _np(x), np.ones(cols), _np(b), True, "bf16")
        g = meq.layer_norm_grad(dy, x, None, r.mean, r.rstd)
        assert g.dweight is None and g.dbias.dtype is torch.float32
        _check_backward(g, _np(dy), _np(x), np.ones(cols), _np(r.mean), _np(r.rstd), 0.0, True, "bf16", "fp32")
        w = _vector(cols, "fp32", 4, 1.0).view(1, cols)
        assert meq.layer_norm_grad(dy, x, w, r.mean, r.rstd, bias=False).dbias is None
        dw, db = torch.empty(cols, dtype=torch.float16, device="cuda"), torch.empty(cols, dtype=torch.float16, device="cuda")
        g = meq.layer_norm_grad(dy, x, w, r.mean, r.rstd, dweight=dw, dbias=db)
        assert g.dweight is dw and g.dbias is db
        _check_backward(g, _np(dy), _np(x), _np(w), _np(r.mean), _np(r.rstd), 0.0, True, "bf16", "fp16")
        assert meq.layer_norm_grad(dy, x, w, r.mean, r.rstd).dweight.shape == w.shape
        empty = torch.empty(0, cols, dtype=torch.bfloat16, device="cuda")
        none = torch.empty(0, device="cuda")
        assert meq.layer_norm(empty, w, eps=EPS).y.shape == (0, cols)
        g = meq.layer_norm_grad(empty, empty, w, none, none)
        assert not g.dweight.any() and not g.dbias.any() and g.dx.shape == (0, cols)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("cols", [33, 256, 1025, 17000])
def test_gradient_against_differences(meq, kind, cols):
    """<gradient, direction> against the 64-bit forward pass a small step to either side, for x, w and b."""
    rows, g = 4, np.random.default_rng(cols)
    x, w, b = _random(rows, cols, "fp32", 1), _vector(cols, "fp32", 2, 1.0), _vector(cols, "fp32", 3, 0.0)
    dy = _random(rows, cols, "fp32", 4)
    r = _forward(meq, kind, x, w, b if kind == "layer" else None)
    got = _backward(meq, kind, dy, x, w, r)

    def loss(x, w, b):
        mu, _, rstd, _ = _statistics(x, kind == "layer")
        return float((((x - mu[:, None]) * rstd[:, None] * w + b) * _np(dy)).sum())

    args = [_np(x), _np(w), _np(b) if kind == "layer" else np.zeros(cols)]
    grads = [_np(got.dx), _np(got.dweight)] + ([_np(got.dbias)] if kind == "layer" else [])
    for i, grad in enumerate(grads):
        u = g.standard_normal(args[i].shape)
        step = 1e-4
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + step * u, args[i] - step * u
        want = (loss(*up) - loss(*down)) / (2 * step)
        # truncation: step^2 / 6 times a third derivative, within 100 times the terms' size; the kernel's own error: T above, summed
        size = float(np.abs(grad * u).sum()) + float(np.abs(_np(dy)).sum()) * 1e-3
        assert abs(float((grad * u).sum()) - want) <= size * (step ** 2 * 100 + (140 + cols / 512) * U), (i, float((grad * u).sum()), want)


@pytest.mark.parametrize("cols", WIDTHS)
def test_results_repeat_and_calls_overlap(meq, cols):
    """The same bits again, from several streams at once, and from a captured graph on new inputs."""
    rows = 600
    w, b = _vector(cols, "fp32", 1, 1.0), _vector(cols, "fp32", 2, 0.0)
    xs, dys = [_random(rows, cols, "bf16", s) for s in (3, 4)], [_random(rows, cols, "bf16", s) for s in (5, 6)]

    def both(x, dy, stream=None):
        r = meq.layer_norm(x, w, b, residual=dy, stream=stream)
        return (r.y, r.h, r.mean, r.rstd) + tuple(meq.layer_norm_grad(dy, r.h, w, r.mean, r.rstd, dh=x, stream=stream))

    want = [both(x, dy) for x, dy in zip(xs, dys)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = [both(x, dy, s) for x, dy, s in zip(xs, dys, streams)]
        torch.cuda.synchronize()
        for a, c in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(a, c))
    x, dy = xs[0].clone(), dys[0].clone()
    graphs, outs = [], []
    for s in streams:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs.append(both(x, dy))
        graphs.append(graph)
    for i in (1, 0):
        x.copy_(xs[i])
        dy.copy_(dys[i])
        for graph, out in zip(graphs, outs):
            graph.replay()
            assert all(torch.equal(p, q) for p, q in zip(out, want[i]))


@pytest.mark.parametrize("cols", [96, 1025, 4096, 17000])
def test_rms_norm_with_a_bias(meq, cols):
    """The C call takes a bias, and its gradient, without a mean too."""
    rows, lib = 40, meq.lib
    x, dy = _random(rows, cols, "bf16", 1), _random(rows, cols, "bf16", 2)
    w, b = _vector(cols, "fp32", 3, 1.0), _vector(cols, "fp32", 4, 0.5)
    y, dx, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda")
    dw, db, work = torch.empty_like(w), torch.empty_like(w), torch.empty(lib.meq_layer_norm_work_floats(rows, cols), device="cuda")
    assert lib.meq_layer_norm(x.data_ptr(), cols, None, 0, 1, rows, cols, w.data_ptr(), b.data_ptr(), 0, EPS, y.data_ptr(), cols, None, 0, None,
                              rstd.data_ptr(), None) == 0
    torch.cuda.synchronize()
    _check_forward(meq.RmsNorm(y, None, rstd), _np(x), _np(w), _np(b), False, "bf16")
    assert lib.meq_layer_norm_grad(dy.data_ptr(), cols, x.data_ptr(), cols, None, 0, 1, rows, cols, w.data_ptr(), 0, None, rstd.data_ptr(), dx.data_ptr(),
                                   cols, dw.data_ptr(), db.data_ptr(), 0, work.data_ptr(), None) == 0
    torch.cuda.synchronize()
    _check_backward(meq.LayerNormGrad(dx, dw, db), _np(dy), _np(x), _np(w), None, _np(rstd), 0.0, False, "bf16", "fp32")
    want = _np(dy).sum(0)
    _within(_np(db), want, _round(want, (96 + rows / 100 + 1) * U * np.abs(_np(dy)).sum(0), "fp32"))
    # dbias alone, and neither
    other = torch.empty_like(w)
    for out in (other.data_ptr(), None):
        assert lib.meq_layer_norm_grad(dy.data_ptr(), cols, x.data_ptr(), cols, None, 0, 1, rows, cols, w.data_ptr(), 0, None, rstd.data_ptr(),
                                       dx.data_ptr(), cols, None, out, 0, work.data_ptr(), None) == 0
    torch.cuda.synchronize()
    assert torch.equal(other, db)


@pytest.mark.parametrize("rows,cols,pad", [(1, 65536, 0), (64, 1024, 0), (65, 1024, 0), (683, 95, 0), (8, 8191, 1), (3, 16400, 0), (2, 20000, 0), (7, 40, 0)])
def test_few_elements_with_and_without_work(meq, rows, cols, pad):
    """Up to 65536 elements a call may do without work, or says that it needs it; the results with it are the same."""
    lib, w = meq.lib, _vector(cols, "fp32", 3, 1.0)
    x, dy = _random(rows, cols, "bf16", 1, pad), _random(rows, cols, "bf16", 2, pad)
    r = meq.layer_norm(x, w, eps=EPS)
    dx, (dw, db) = _matrix(rows, cols, "bf16", pad), torch.empty(2, cols, device="cuda")
    args = (dy.data_ptr(), cols + pad, x.data_ptr(), cols + pad, None, 0, 1, rows, cols, w.data_ptr(), 0, r.mean.data_ptr(), r.rstd.data_ptr(), dx.data_ptr(),
            cols + pad, dw.data_ptr(), db.data_ptr(), 0)
    status = lib.meq_layer_norm_grad(*args, None, None)
    assert status == (1 if rows * cols > 65536 or cols > 16384 else 0)
    if status:
        assert b"work" in lib.meq_last_error(None)
    torch.cuda.synchronize()
    first = dx.clone(), dw.clone(), db.clone()
    work = torch.full((lib.meq_layer_norm_work_floats(rows, cols),), float("nan"), device="cuda")
    assert lib.meq_layer_norm_grad(*args, work.data_ptr(), None) == 0
    torch.cuda.synchronize()
    _check_backward(meq.LayerNormGrad(dx, dw, db), _np(dy), _np(x), _np(w), _np(r.mean), _np(r.rstd), 0.0, True, "bf16", "fp32")
    if not status:
        assert all(torch.equal(p, q) for p, q in zip(first, (dx, dw, db)))
    g = meq.layer_norm_grad(dy, x, w, r.mean, r.rstd)   # the binding finds out by itself; here dx is contiguous
    _check_backward(g, _np(dy), _np(x), _np(w), _np(r.mean), _np(r.rstd), 0.0, True, "bf16", "fp32")


def test_numbers_of_other_kinds(meq):
    x, w = torch.randn(3, 8, device="cuda"), torch.ones(8, device="cuda")
    assert torch.equal(meq.rms_norm(x, w, eps=np.float32(1e-6)).y, meq.rms_norm(x, w).y)
    t = torch.tensor([1, 2], device="cuda")
    assert torch.equal(meq.embedding(t, x, scale=np.float64(2)), meq.embedding(t, x, scale=2))


def test_refusals(meq):
    x, w, v = torch.zeros(4, 8, device="cuda"), torch.ones(8, device="cuda"), torch.zeros(4, device="cuda")
    half, wide = x.half(), torch.zeros(4, 16, device="cuda")
    bad = [lambda: meq.layer_norm(x[0], w), lambda: meq.layer_norm(x.double(), w), lambda: meq.layer_norm(x.T, w), lambda: meq.layer_norm(x.cpu(), w),
           lambda: meq.layer_norm(x, w[:4]), lambda: meq.layer_norm(x, w.double()), lambda: meq.layer_norm(x, w, w.half()),
           lambda: meq.layer_norm(x, wide[0, ::2]), lambda: meq.layer_norm(x, w, residual=half), lambda: meq.layer_norm(x, w, residual=x[:2]),
           lambda: meq.layer_norm(x, w, h=x), lambda: meq.layer_norm(x, w, y=half), lambda: meq.layer_norm(x, w, y=x[:1].expand(4, 8)),
           lambda: meq.layer_norm(wide[:, ::2], w), lambda: meq.layer_norm_grad(x, half, w, v, v), lambda: meq.layer_norm_grad(x, x, w, v[:2], v),
           lambda: meq.layer_norm_grad(x, x, w, v, v.double()), lambda: meq.layer_norm_grad(x, x, w, v, v, dh=x[:2]),
           lambda: meq.layer_norm_grad(x, x, w, v, v, dx=half), lambda: meq.layer_norm_grad(x, x, w, v, v, dweight=w.half()[:4]),
           lambda: meq.layer_norm_grad(x, x, w, v, v, dweight=w.clone(), dbias=w.half()), lambda: meq.layer_norm_grad(x, x, w, None, v)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(i)
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(meq.MeqError):
            meq.layer_norm(x, w, eps=eps)
    with pytest.raises(meq.MeqError):
        meq.layer_norm(x, w, residual=x, y=wide[:, :8], h=wide[:, :8])


@pytest.mark.parametrize("cols", WIDTHS)
def test_a_norm_over_its_input_leaves_no_h(meq, cols):
    """y = x without a residual: what was normalised is gone, so there is none to take a gradient from."""
    rows, w, b = 37, _vector(cols, "fp32", 1, 1.0), _vector(cols, "fp32", 2, 0.0)
    x, res, dy = (_random(rows, cols, "bf16", s) for s in (3, 4, 5))
    want, rms = meq.layer_norm(x, w, b), meq.rms_norm(x, w)
    assert want.h is x and rms.h is x
    for same in (lambda t: t, lambda t: t.view(rows, cols)):  # the same tensor, and another of the same memory
        a = x.clone()
        got = meq.layer_norm(a, w, b, y=same(a))
        assert torch.equal(got.y, want.y) and got.h is None
        with pytest.raises(ValueError, match="h must be given"):
            meq.layer_norm_grad(dy, got.h, w, got.mean, got.rstd)
        a = x.clone()
        got = meq.rms_norm(a, w, y=same(a))
        assert torch.equal(got.y, rms.y) and got.h is None
        with pytest.raises(ValueError, match="h must be given"):
            meq.rms_norm_grad(dy, got.h, w, got.rstd)
    assert meq.layer_norm(x, w, b, y=dy).h is x
    # with a residual the sum is kept, whatever y takes the place of
    kept = meq.layer_norm(x, w, b, residual=res).h
    a, c = x.clone(), res.clone()
    assert torch.equal(meq.layer_norm(a, w, b, residual=res, y=a).h, kept) and torch.equal(meq.layer_norm(x, w, b, residual=c, y=c).h, kept)
    none = torch.empty(0, cols, dtype=torch.bfloat16, device="cuda")  # nothing is overwritten
    assert meq.layer_norm(none, w, b, y=none).h is none


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(5, 40), (5, 96), (4, 1025), (3, 4096), (700, 128), (300, 1025), (300, 4096), (40, 9000), (5, 17000)])
def test_tiny_rows_that_vary(meq, kind, dtype, rows, cols):
    """rstd near 3e20 and gradients as large: finite whatever the rows' length, though rstd's square is not."""
    x = _random(rows, cols, dtype, 1, spread=3e-21)
    dy, dh, w = _random(rows, cols, dtype, 2), _random(rows, cols, dtype, 3), _vector(cols, "fp32", 4, 1.0)
    r = meq.layer_norm(x, w, eps=1e-44) if kind == "layer" else meq.rms_norm(x, w, eps=1e-44)
    assert bool((r.rstd > 1e19).all()) and bool(r.rstd.isfinite().all())
    for more in (None, dh):
        g = _backward(meq, kind, dy, x, w, r, dh=more)
        _check_backward(g, _np(dy), _np(x), _np(w), _np(r.mean) if kind == "layer" else None, _np(r.rstd), 0.0 if more is None else _np(dh),
                        kind == "layer", dtype, "fp32")


# The longest aligned rows that a group of warps holds, and the next, per type: backward with dh, layer norm's and RMS norm's.
LIMITS = [("bf16", 13312), ("bf16", 13320), ("fp16", 14336), ("bf16", 16384), ("bf16", 16392), ("bf16", 16377), ("bf16", 16378),
          ("fp32", 9216), ("fp32", 9220), ("fp32", 9213), ("fp32", 9214), ("fp32", 10240), ("fp32", 10244), ("fp32", 10237), ("fp32", 10238)]


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("rows", [3, 40])
@pytest.mark.parametrize("dtype,cols", LIMITS)
def test_either_side_of_the_longest_rows_in_registers(meq, kind, rows, dtype, cols):
    x, res, dy, dh = (_random(rows, cols, dtype, s) for s in (1, 2, 3, 4))
    w, b = _vector(cols, "fp32", 5, 1.0), _vector(cols, "fp32", 6, 0.0)
    r = _forward(meq, kind, x, w, b if kind == "layer" else None, residual=res)
    _check_forward(r, _np(r.h), _np(w), _np(b) if kind == "layer" else 0.0, kind == "layer", dtype)
    for more in (None, dh):
        g = _backward(meq, kind, dy, r.h, w, r, dh=more)
        _check_backward(g, _np(dy), _np(r.h), _np(w), _np(r.mean) if kind == "layer" else None, _np(r.rstd), 0.0 if more is None else _np(dh),
                        kind == "layer", dtype, "fp32")


@pytest.mark.parametrize("weight_type", ["fp32", "bf16"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cols", [40, 768, 1025, 4096, 17000])
def test_weights_that_start_anywhere(meq, cols, dtype, weight_type):
    """Weight, bias and their gradients as parts of one vector, each an element further: the bits of aligned ones."""
    rows, held = 37, torch.zeros(4 * cols + 16, dtype=DT[weight_type], device="cuda")
    x, dy = _random(rows, cols, dtype, 1), _random(rows, cols, dtype, 2)
    w, b = _vector(cols, weight_type, 3, 1.0), _vector(cols, weight_type, 4, 0.0)
    w1, b1, dw1, db1 = (held[i * (cols + 1) + 1:][:cols] for i in range(4))
    w1.copy_(w)
    b1.copy_(b)
    want, got = meq.layer_norm(x, w, b), meq.layer_norm(x, w1, b1)
    assert torch.equal(got.y, want.y) and torch.equal(got.mean, want.mean) and torch.equal(got.rstd, want.rstd)
    want, got = (meq.layer_norm_grad(dy, x, a, got.mean, got.rstd, dweight=p, dbias=q) for a, p, q in ((w, None, None), (w1, dw1, db1)))
    assert got.dweight is dw1 and all(torch.equal(p, q) for p, q in zip(got, want))


def test_rows_that_a_32_bit_offset_does_not_reach(meq):
    """Three rows 1.2e9 elements apart, read and written in buffers of their own."""
    rows, apart = 3, 1200000000

    def far():
        return torch.empty(2 * apart + 20000, dtype=torch.bfloat16, device="cuda")

    buffers = [far() for _ in range(4)]
    for cols in (96, 1025, 4096, 17000):
        def view(t, like=None):
            v = t.as_strided((rows, cols), (apart, 1))
            return v if like is None else v.copy_(like)

        x, res, dy = (_random(rows, cols, "bf16", s) for s in (1, 2, 3))
        w, b = _vector(cols, "fp32", 4, 1.0), _vector(cols, "fp32", 5, 0.0)
        want = meq.layer_norm(x, w, b, residual=res)
        held = view(buffers[1], res)
        got = meq.layer_norm(view(buffers[0], x), w, b, residual=held, y=view(buffers[2]), h=view(buffers[3]))
        assert torch.equal(got.h, want.h)
        _check_forward(got, _np(got.h), _np(w), _np(b), True, "bf16")
        g = meq.layer_norm_grad(view(buffers[0], dy), got.h, w, want.mean, want.rstd, dh=held, dx=view(buffers[2]))
        _check_backward(g, _np(dy), _np(want.h), _np(w), _np(want.mean), _np(want.rstd), _np(res), True, "bf16", "fp32")
