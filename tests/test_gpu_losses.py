"""Token log-probabilities, the policy loss and the preference loss against plain 64-bit arithmetic.

Tolerances. The sum of exponentials has a relative error of at most 2^-18: 2^-22 for each exponential,
2^-24 for each of the at most 50 additions on the way of a term (32 in a thread, 15 in the trees), and the
rounding of z - max, which weighs d exp(-d) <= 0.37 with d = max - z. So
  T(logp) = 2^-18 + 2^-22 (|logp| + |z_t - max| + 1).
A gradient c (onehot - p) adds 2^-17 |c| p, the error of c, which is the slope's magnitude times 2 T(logp)
and a few roundings, and half an ulp of its type (2^-8 of a bf16 value, 2^-11 of an fp16 one or 2^-25 below
its normal range, 2^-24 of an fp32 one).
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF_ULP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
LEAST = {"fp32": 1e-37, "bf16": 1e-37, "fp16": 2.0 ** -25}


@pytest.fixture(scope="module")
def meq():
    import __graft_entry__

    __graft_entry__.build()
    from paper_2609_35701_gb300 import meq as m

    return m


def _np(t):
    return t.detach().cpu().double().numpy()


def _matrix(rows, cols, dtype, pad=0, shift=0, fill=None):
    """A CUDA matrix whose rows are `pad` elements apart and that starts `shift` elements into its allocation."""
    flat = torch.zeros(rows * (cols + pad) + shift, dtype=DT[dtype], device="cuda")
    if fill is not None:
        flat.fill_(fill)
    return flat[shift:].view(rows, cols + pad)[:, :cols]


def _tokens(rows, cols, dtype, seed, pad=0, shift=0, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    z = spread * torch.randn(rows, cols, generator=g)
    t = torch.randint(0, cols, (rows,), generator=g)
    z[torch.arange(rows), t] += 4.0
    m = _matrix(rows, cols, dtype, pad, shift)
    m.copy_(z)
    return m, t.cuda(), g


def _rows64(z, t):
    """(logp, softmax, |z_t - max|) in 64 bits."""
    z = _np(z)
    top = z.max(1, keepdims=True)
    e = np.exp(z - top)
    s = e.sum(1, keepdims=True)
    zt = np.take_along_axis(z, np.maximum(_np(t).astype(np.int64), 0)[:, None], 1)
    return (zt - top - np.log(s))[:, 0], e / s, np.abs(zt - top)[:, 0]


def _tol(logp, dist):
    return 2.0 ** -18 + 2.0 ** -22 * (np.abs(logp) + dist + 1)


def _check_grad(got, c, dc, p, t, dtype):
    """got against c (onehot - p), c off by at most dc."""
    want = -c[:, None] * p
    np.put_along_axis(want, t[:, None], np.take_along_axis(want, t[:, None], 1) + c[:, None], 1)
    tol = np.abs(c)[:, None] * p * 2.0 ** -17 + dc[:, None] * (p + (want != -c[:, None] * p)) + LEAST[dtype]
    tol = tol + HALF_ULP[dtype] * (np.abs(want) + tol)
    assert (np.abs(got - want) <= tol).all(), np.max(np.abs(got - want) / tol)


SIZES = [(5, 1, 0, 0), (5, 2, 1, 1), (3, 7, 0, 0), (4, 8, 0, 3), (4, 9, 0, 0), (6, 63, 2, 1), (3, 1000, 0, 0), (5, 4095, 1, 0),
         (3, 4096, 0, 1), (3, 4097, 7, 5), (2, 32000, 0, 0), (3, 50001, 0, 0), (2, 151936, 128, 0), (400, 4111, 0, 0)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,cols,pad,shift", SIZES)
def test_logprobs(meq, dtype, rows, cols, pad, shift):
    z, t, _ = _tokens(rows, cols, dtype, rows * 1000 + cols, pad, shift)
    t[rows // 2] = -100
    want, _, dist = _rows64(z, t)
    r = meq.token_logprobs(z, t)
    scored = _np(t) >= 0
    zt = _np(z)[np.arange(rows), np.maximum(_np(t).astype(int), 0)]
    assert (np.abs(_np(r.logp) - want) <= _tol(want, dist))[scored].all()
    lse = zt - want
    assert (np.abs(_np(r.lse) - lse) <= _tol(want, dist) + 2.0 ** -22 * np.abs(lse))[scored].all()
    assert not _np(r.logp)[~scored].any() and not _np(r.lse)[~scored].any()


# more than the registers of a cluster hold, in each element size
LARGE = [("fp32", 3, 270001, 0, 0), ("bf16", 2, 530001, 3, 1), ("fp16", 2, 524288, 0, 0), ("fp32", 2, 1048583, 0, 1)]


@pytest.mark.parametrize("dtype,rows,cols,pad,shift", LARGE)
def test_logprobs_of_rows_that_no_cluster_holds(meq, dtype, rows, cols, pad, shift):
    z, t, _ = _tokens(rows, cols, dtype, 3, pad, shift)
    want, _, dist = _rows64(z, t)
    assert (np.abs(_np(meq.token_logprobs(z, t).logp) - want) <= _tol(want, dist)).all()


CLIP_LOW, CLIP_HIGH = 0.2, 0.28


def _policy_inputs(z, t, g, kl):
    return _policy_inputs_at(_rows64(z, t)[0], g, kl)


def _policy_inputs_at(logp, g, kl):
    n = len(logp)
    d = 0.3 * torch.randn(n, generator=g).double().numpy()
    for edge in (1 - CLIP_LOW, 1 + CLIP_HIGH):  # no ratio where rounding decides whether it is clipped
        d = np.where(np.abs(np.exp(d) - edge) < 1e-3, d + 5e-3, d)
    f = lambda x: torch.tensor(x, dtype=torch.float32).cuda()  # noqa: E731
    adv = torch.randn(n, generator=g).cuda()
    w = (torch.rand(n, generator=g) + 0.1).cuda() / n
    w[::5] = 0.0
    w[0] = 0.5 / n
    ref = f(logp - 0.4 * torch.randn(n, generator=g).double().numpy()) if kl else None
    return f(logp - d), adv, w, ref


def _policy64(logp, old, adv, w, ref, kl):
    ratio = np.exp(logp - old)
    plain, bounded = ratio * adv, np.clip(ratio, 1 - CLIP_LOW, 1 + CLIP_HIGH) * adv
    cut = plain > bounded
    surrogate = -np.minimum(plain, bounded)
    slope, k3, size = np.where(cut, 0.0, -plain), np.zeros_like(logp), np.abs(plain)
    if kl:
        d = ref - logp
        k3 = np.expm1(d) - d
        slope = slope - kl * np.expm1(d)
        size = size + kl * (np.exp(d) + 1)
    terms = np.stack([w * (surrogate + kl * k3), w * surrogate, w * k3, w * cut])
    return terms, w * slope, np.abs(w) * size


def _check_policy(meq, z, t, g, kl, dtype, grad, scale=None):
    old, adv, w, ref = _policy_inputs(z, t, g, kl)
    gs = 1.0 if scale is None else float(scale)
    logp, p, dist = _rows64(z, t)
    r = meq.policy_loss(z, t, old, adv, w, ref, CLIP_LOW, CLIP_HIGH, kl, grad=grad, grad_scale=scale)
    scored = (_np(t) >= 0) & (_np(w) != 0)
    tol = _tol(logp, dist)
    assert (np.abs(_np(r.logp) - np.where(scored, logp, 0)) <= tol).all()
    ref64 = None if ref is None else _np(ref)
    terms, c, size = _policy64(logp, _np(old), _np(adv), np.where(scored, _np(w), 0), ref64, kl)
    # a term moves by its slope, at most `size`, times the error of logp, and by its own roundings
    # (of the surrogate, and of d as a part of exp(d) - d - 1)
    slack = (size * (2 * tol + 2.0 ** -20) + 2.0 ** -20 * np.abs(terms).sum(0)).sum()
    got = _np(r.sums)
    assert (np.abs(got - terms.sum(1)) <= slack * (1 + (1 / kl if kl else 0)) + 1e-12).all(), (got, terms.sum(1), slack)
    assert float(r.loss) == float(r.sums[0])
    if r.grad is not None:
        assert r.grad.shape == z.shape and r.grad.dtype is z.dtype
        _check_grad(_np(r.grad), c * gs, size * gs * (2 * tol + 2.0 ** -20), np.where(scored[:, None], p, 0), np.maximum(_np(t).astype(np.int64), 0), dtype)
        assert not _np(r.grad)[~scored].any()
    return r


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("kl", [0.0, 0.05])
@pytest.mark.parametrize("rows,cols,pad,shift", SIZES)
def test_policy_loss(meq, dtype, kl, rows, cols, pad, shift):
    z, t, g = _tokens(rows, cols, dtype, rows * 1000 + cols, pad, shift)
    if rows > 3:
        t[2] = -1
    scale = torch.tensor([512.0], device="cuda") if dtype == "fp16" else None
    _check_policy(meq, z, t, g, kl, dtype, True, scale)


@pytest.mark.parametrize("dtype,rows,cols,pad,shift", LARGE)
def test_policy_loss_of_rows_that_no_cluster_holds(meq, dtype, rows, cols, pad, shift):
    z, t, g = _tokens(rows, cols, dtype, 3, pad, shift)
    _check_policy(meq, z, t, g, 0.05, dtype, True)


# many long rows: one CTA per row, then clusters of 2, 4 and 8, aligned and not
STREAMED = [("bf16", 700, 20011, 0, 0), ("bf16", 310, 32000, 0, 0), ("fp16", 330, 57345, 1, 3), ("fp32", 320, 28672, 0, 0),
            ("fp32", 307, 50001, 2, 1), ("bf16", 310, 60001, 5, 0), ("bf16", 305, 151936, 0, 0), ("fp16", 305, 200003, 0, 1),
            ("fp32", 304, 151936, 64, 0), ("fp32", 304, 262147, 0, 3), ("bf16", 304, 800003, 0, 0)]


@pytest.mark.parametrize("dtype,rows,cols,pad,shift", STREAMED)
@pytest.mark.parametrize("scored", [1.0, 0.6, 0.01])
def test_many_long_rows(meq, dtype, rows, cols, pad, shift, scored):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    z = _matrix(rows, cols, dtype, pad, shift)
    z.copy_(3.0 * torch.randn(rows, cols, generator=g, device="cuda"))
    t = torch.randint(0, cols, (rows,), generator=g, device="cuda")
    t[:4] = torch.tensor([0, cols - 1, 1, cols // 2], device="cuda")
    skip = torch.rand(rows, generator=g, device="cuda") >= scored
    skip[0] = False
    keep = torch.where(skip, -100, t)
    logp64, dist = torch.zeros(rows, dtype=torch.float64, device="cuda"), torch.zeros(rows, dtype=torch.float64, device="cuda")
    for i in range(0, rows, 64):
        x = z[i:i + 64].double()
        zt = x.gather(1, t[i:i + 64, None])[:, 0]
        logp64[i:i + 64], dist[i:i + 64] = zt - torch.logsumexp(x, 1), (zt - x.amax(1)).abs()
    logp, dist = _np(logp64), _np(dist)
    tol = _tol(logp, dist)
    on = ~_np(skip).astype(bool)
    r = meq.token_logprobs(z, keep)
    assert (np.abs(_np(r.logp) - logp) <= tol)[on].all() and not _np(r.logp)[~on].any()
    old, adv, w, ref = _policy_inputs_at(logp, torch.Generator().manual_seed(1), 0.05)
    r = meq.policy_loss(z, keep, old, adv, w, ref, CLIP_LOW, CLIP_HIGH, 0.05, grad=True)
    on &= _np(w) != 0
    assert (np.abs(_np(r.logp) - logp) <= tol)[on].all() and not _np(r.logp)[~on].any()
    _, c, size = _policy64(logp, _np(old), _np(adv), np.where(on, _np(w), 0), _np(ref), 0.05)
    c, dc = torch.tensor(c).cuda(), torch.tensor(size * (2 * tol + 2.0 ** -20)).cuda()
    for i in range(0, rows, 64):
        p = torch.softmax(z[i:i + 64].double(), 1)
        want = -c[i:i + 64, None] * p
        hit = torch.zeros_like(p).scatter_(1, t[i:i + 64, None], 1.0)
        want += c[i:i + 64, None] * hit
        bound = c[i:i + 64, None].abs() * p * 2.0 ** -17 + dc[i:i + 64, None] * (p + hit) + LEAST[dtype]
        bound += HALF_ULP[dtype] * (want.abs() + bound)
        assert ((r.grad[i:i + 64].double() - want).abs() <= bound).all(), i
    assert not r.grad[torch.tensor(~on).cuda()].any()
    again = meq.policy_loss(z, keep, old, adv, w, ref, CLIP_LOW, CLIP_HIGH, 0.05, grad=z)  # in place
    assert torch.equal(again.grad, r.grad) and torch.equal(again.sums, r.sums)


# many rows that a warp holds (up to 4 KB), of one to eight 16-byte pieces per lane, and the first that it does not
SHORT = [("bf16", 20000, 256, 0, 0), ("bf16", 9001, 250, 1, 3), ("fp32", 17000, 100, 0, 1), ("fp16", 9000, 1000, 0, 0),
         ("fp32", 8193, 1021, 3, 0), ("bf16", 6000, 2034, 0, 0), ("bf16", 4100, 2035, 2, 0), ("fp16", 30000, 3, 0, 1)]


@pytest.mark.parametrize("dtype,rows,cols,pad,shift", SHORT)
def test_many_short_rows(meq, dtype, rows, cols, pad, shift):
    z, t, g = _tokens(rows, cols, dtype, rows + cols, pad, shift)
    t[::7] = -1
    t[5000:5100] = -100
    r = _check_policy(meq, z, t, g, 0.05, dtype, True)
    logp, _, dist = _rows64(z, t)
    on = _np(t) >= 0
    one = meq.token_logprobs(z, t)
    zt = _np(z)[np.arange(rows), np.maximum(_np(t).astype(int), 0)]
    assert (np.abs(_np(one.logp) - logp) <= _tol(logp, dist))[on].all() and not _np(one.logp)[~on].any() and not _np(one.lse)[~on].any()
    assert (np.abs(_np(one.lse) - (zt - logp)) <= _tol(logp, dist) + 2.0 ** -22 * np.abs(zt - logp))[on].all()
    args = (t, one.logp, torch.ones(rows, device="cuda"), None, one.logp)
    a = meq.policy_loss(z, *args, kl_coef=0.1, grad=True)
    b = meq.policy_loss(z, *args, kl_coef=0.1, grad=z)  # in place
    assert torch.equal(a.grad, b.grad) and torch.equal(a.sums, b.sums) and torch.equal(a.logp, b.logp)
    assert r.grad.shape == b.grad.shape


@pytest.mark.parametrize("dtype,cols,pad,shift", [("bf16", 256, 0, 0), ("fp32", 301, 1, 1), ("fp16", 1500, 0, 0), ("bf16", 2035, 2, 0)])
def test_preference_of_many_short_rows(meq, dtype, cols, pad, shift):
    lengths = [700, 1, 0, 333, 1024, 90, 5, 2001]
    test_preference_loss(meq, dtype, lengths, cols, pad, shift, 0.1)


@pytest.mark.parametrize("scored", ["none", "one", "runs"])
@pytest.mark.parametrize("cols", [25000, 100000])
def test_masks_that_leave_little(meq, cols, scored):
    """No row scored, one, or long runs of each, among many long rows."""
    rows = 1300
    g = torch.Generator(device="cuda").manual_seed(cols)
    z = torch.randn(rows, cols, generator=g, device="cuda").bfloat16()
    t = torch.full((rows,), -100, device="cuda")
    if scored == "one":
        t[777] = 5
    elif scored == "runs":
        t[:300], t[700:705], t[1299] = 3, 0, cols - 1
    on = t >= 0
    want = torch.where(on, torch.stack([torch.log_softmax(z[i].double(), 0)[max(int(t[i]), 0)] for i in range(rows)]), 0.0)
    r = meq.token_logprobs(z, t)
    assert ((r.logp.double() - want).abs() <= 2.0 ** -17).all() and not r.logp[~on].any()
    zero = torch.zeros(rows, device="cuda")
    r = meq.policy_loss(z, t, r.logp, zero + 1, zero + 1, grad=True)   # ratios of 1 but for rounding: the loss counts the scored rows
    assert abs(float(r.loss) + float(on.sum())) <= 2.0 ** -16 * float(on.sum())
    assert not r.grad[~on].any() and bool((r.grad[on] != 0).any(1).all() if on.any() else True)


@pytest.mark.parametrize("dtype,rows,cols", [("bf16", 700, 40003), ("fp32", 330, 50001), ("bf16", 305, 151936)])
@pytest.mark.parametrize("place", ["apart", "in place"])
def test_a_wait_that_runs_out_gives_nan(meq, dtype, rows, cols, place):
    """The data of one row never comes, the waits' limit is 20 ms: the kernel ends, every row of that block (or cluster of
    blocks) is NaN in all its results, every other row is right, and so is the next call."""
    g = torch.Generator(device="cuda").manual_seed(cols)
    z = _matrix(rows, cols, dtype)
    z.copy_(torch.randn(rows, cols, generator=g, device="cuda"))
    t = torch.randint(0, cols, (rows,), generator=g, device="cuda")
    t[::3] = -1
    row = 103
    assert int(t[row]) >= 0
    adv, w = torch.linspace(0.5, 1.5, rows, device="cuda"), torch.full((rows,), 1.0 / rows, device="cuda")
    plain = meq.token_logprobs(z, t)
    good = meq.policy_loss(z, t, plain.logp, adv, w, grad=True)
    assert bool(torch.isfinite(good.loss)) and bool(torch.isfinite(good.grad).all())
    try:
        meq.debug_loss_wait(20.0, row)
        stats = meq.token_logprobs(z, t)
        bad = meq.policy_loss(z, t, plain.logp, adv, w, grad=z.clone() if place == "apart" else z)
        torch.cuda.synchronize()
    finally:
        meq.debug_loss_wait()
    for got, want in ((stats.logp, plain.logp), (stats.lse, plain.lse), (bad.logp, good.logp), (bad.grad, good.grad)):
        lost = torch.isnan(got).view(rows, -1)
        assert bool((lost.any(1) == lost.all(1)).all())
        lost = lost.any(1)
        assert bool(lost[row]) and int(lost.sum()) < rows // 4
        at = lost.nonzero()[:, 0]
        assert at.numel() < 2 or len(set((at[1:] - at[:-1]).tolist())) == 1   # a block's rows lie a fixed number apart
        assert torch.equal(got[~lost], want[~lost])
    assert bool(torch.isnan(bad.sums).all())
    if place == "in place":
        return
    again = meq.policy_loss(z, t, plain.logp, adv, w, grad=True)
    assert torch.equal(again.grad, good.grad) and torch.equal(again.sums, good.sums)


@pytest.mark.parametrize("dtype,rows,cols,pad,shift", [c for c in STREAMED if c[2] not in (20011, 262147)])
def test_many_long_rows_without_a_gradient(meq, dtype, rows, cols, pad, shift):
    """The loss alone is the same, bit for bit, as with its gradient (which the tests above compare with 64 bits)."""
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    z = _matrix(rows, cols, dtype, pad, shift)
    z.copy_(3.0 * torch.randn(rows, cols, generator=g, device="cuda"))
    t = torch.randint(-cols // 2, cols, (rows,), generator=g, device="cuda")
    old, adv = torch.full((rows,), -math.log(cols) - 4.0, device="cuda"), torch.randn(rows, generator=g, device="cuda")
    keep = z.clone()
    with_grad = meq.policy_loss(z, t, old, adv, ref_logp=old, kl_coef=0.1, grad=True)
    alone = [meq.policy_loss(z, t, old, adv, ref_logp=old, kl_coef=0.1) for _ in range(2)]
    for r in alone:
        assert r.grad is None and torch.equal(r.sums, with_grad.sums) and torch.equal(r.logp, with_grad.logp)
    assert bool(torch.isfinite(with_grad.loss)) and torch.equal(z, keep)


def test_calls_from_several_threads(meq):
    """Four host threads, a stream each, calls of every form and refused calls among them: the results are those of one
    thread, and a refusal's text is that of the thread's own call."""
    import threading

    shapes = [("bf16", 400, 40003), ("fp32", 9, 4111), ("fp16", 3000, 250), ("bf16", 310, 151936)]
    data, want = [], []

    def calls(i, stream=None):
        z, t, v, starts = data[i]
        out = list(meq.token_logprobs(z, t, stream=stream)) + list(meq.policy_loss(z, t, v, v + 1, grad=True, stream=stream))
        r = meq.preference_loss(z, t, starts, v, grad=True, stream=stream)
        return out + [r.loss, r.margins, r.logp, r.grad]

    for i, (dtype, rows, cols) in enumerate(shapes):
        z, t, _ = _tokens(rows, cols, dtype, i)
        data.append((z, t, torch.full((rows,), -9.0, device="cuda"), torch.tensor([0, rows // 3, rows], device="cuda")))
        want.append([x.clone() for x in calls(i)])
    torch.cuda.synchronize()
    failures, start = [], threading.Barrier(len(shapes))

    def work(i):
        try:
            stream = torch.cuda.Stream()
            start.wait()
            for _ in range(15):
                got = calls(i, stream)
                name = ("clip_low", "kl_coef")[i % 2]
                with pytest.raises(meq.MeqError, match=name):
                    meq.policy_loss(*data[i][:2], data[i][2], data[i][2], **{name: -1.0}, stream=stream)
                stream.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(got, want[i]))
        except BaseException as e:  # noqa: BLE001 - reported by the main thread
            failures.append((i, e))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(shapes))]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not failures, failures


def test_a_wait_that_runs_out_in_the_preference_loss(meq):
    rows, cols = 700, 40003
    z = torch.randn(rows, cols, device="cuda").bfloat16()
    t, starts, ref = torch.full((rows,), 5, device="cuda"), torch.tensor([0, 200, 350, 500, 700], device="cuda"), torch.zeros(rows, device="cuda")
    try:
        meq.debug_loss_wait(20.0, 103)
        r = meq.preference_loss(z, t, starts, ref, grad=True)
        torch.cuda.synchronize()
    finally:
        meq.debug_loss_wait()
    assert bool(torch.isnan(r.loss)) and bool(torch.isnan(r.margins[0])) and bool(torch.isnan(r.grad[103]).all())
    assert bool(torch.isnan(r.logp[103]))
    with pytest.raises(meq.MeqError):
        meq.debug_loss_wait(-1.0)


def test_offsets_past_32_bits_in_a_long_batch(meq):
    """490000 rows of 24000 equal logits, 23.5 GB: log-probabilities of -log(24000), a gradient of 1/24000 each."""
    rows, cols = 490000, 24000
    z = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    t = torch.arange(rows, device="cuda") % cols
    t[::3] = -1
    on = t >= 0
    r = meq.token_logprobs(z, t)
    assert ((r.logp.double() + math.log(cols)).abs()[on] <= 2.0 ** -17).all() and not r.logp[~on].any()
    zero = torch.zeros(rows, device="cuda")
    r = meq.policy_loss(z, t, r.logp, zero + 1, zero + 1, grad=z)
    assert abs(float(r.loss) + float(on.sum())) <= 2.0 ** -16 * float(on.sum())
    # c = -1: softmax - onehot
    assert not z[~on].any()
    rowsum = torch.cat([x.float().sum(1) for x in z.split(20000)])
    assert (rowsum[on].abs() < 2.0 ** -7).all()   # 23999 bf16 values of 1/24000 and one of 1/24000 - 1
    assert (z.gather(1, t.clamp(min=0)[:, None])[:, 0][on].float() + 1 < 2.0 ** -8).all()


@pytest.mark.parametrize("cols,pad,gpad,gshift", [(1001, 0, 0, 1), (1001, 0, 1, 0), (1000, 8, 0, 3), (4099, 1, 6, 0)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gradient_rows_at_other_offsets_than_the_logits(meq, dtype, cols, pad, gpad, gshift):
    z, t, g = _tokens(7, cols, dtype, 11, pad, 0)
    grad = _matrix(7, cols, dtype, gpad, gshift, fill=77.0)
    whole = grad.as_strided((grad.untyped_storage().nbytes() // grad.element_size(),), (1,), 0)
    r = _check_policy(meq, z, t, g, 0.05, dtype, grad)
    assert r.grad is grad
    inside = torch.zeros(whole.numel(), dtype=torch.bool, device="cuda")
    inside.as_strided(grad.shape, grad.stride(), grad.storage_offset())[:] = True
    assert (whole[~inside] == 77.0).all()  # nothing beside the rows is written


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("cols", [1003, 32000, 600011])
def test_gradient_in_place_of_the_logits(meq, dtype, cols):
    z, t, g = _tokens(4, cols, dtype, 5, 3, 1)
    old, adv, w, ref = _policy_inputs(z, t, g, 0.05)
    apart = meq.policy_loss(z, t, old, adv, w, ref, CLIP_LOW, CLIP_HIGH, 0.05, grad=True)
    here = meq.policy_loss(z, t, old, adv, w, ref, CLIP_LOW, CLIP_HIGH, 0.05, grad=z)
    assert torch.equal(apart.grad, z) and torch.equal(apart.sums, here.sums) and torch.equal(apart.logp, here.logp)


def _pref_inputs(lengths, cols, dtype, seed, pad=0, shift=0):
    n = sum(lengths)
    z, t, g = _tokens(n, cols, dtype, seed, pad, shift)
    w = (torch.rand(n, generator=g) < 0.7).float().cuda()
    starts = torch.tensor([0] + list(np.cumsum(lengths)), dtype=torch.int64, device="cuda")
    logp, _, _ = _rows64(z, t)
    ref = torch.tensor(logp - 0.3 * torch.randn(n, generator=g).double().numpy(), dtype=torch.float32).cuda()
    return z, t, w, starts, ref, logp


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("lengths,cols,pad,shift", [([1, 1], 9, 0, 0), ([3, 0], 100, 0, 0), ([0, 0], 5, 0, 0), ([0, 4, 2, 7], 33, 1, 1),
                                                    ([40, 31, 300, 2, 1, 1], 1001, 0, 0), ([3, 4], 50001, 0, 0),
                                                    ([2, 2], 280001, 0, 1)])
@pytest.mark.parametrize("smoothing", [0.0, 0.1])
def test_preference_loss(meq, dtype, lengths, cols, pad, shift, smoothing):
    beta = 0.4
    if sum(lengths) == 0:  # every answer is empty: no margin, log 2
        z = torch.zeros(0, cols, dtype=DT[dtype], device="cuda")
        r = meq.preference_loss(z, torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda"),
                                torch.zeros(0, device="cuda"), beta=beta, label_smoothing=smoothing, grad=True)
        assert abs(float(r.loss) - math.log(2)) < 1e-6 and float(r.margins[0]) == 0.0
        return
    z, t, w, starts, ref, logp = _pref_inputs(lengths, cols, dtype, 17, pad, shift)
    scale = torch.tensor([64.0], device="cuda") if dtype == "fp16" else None
    gs = 64.0 if dtype == "fp16" else 1.0
    r = meq.preference_loss(z, t, starts, ref, w, beta=beta, label_smoothing=smoothing, grad=True, grad_scale=scale)
    _, p, dist = _rows64(z, t)
    tol = _tol(logp, dist)
    pairs, at = len(lengths) // 2, np.concatenate([[0], np.cumsum(lengths)])
    d = _np(w) * (logp - _np(ref))
    c, dc, total, slack = np.zeros_like(logp), np.zeros_like(logp), 0.0, 0.0
    for j in range(pairs):
        a, b, e = at[2 * j:2 * j + 3]
        x = beta * (d[a:b].sum() - d[b:e].sum())
        dx = beta * (_np(w)[a:e] * tol[a:e]).sum() + 2.0 ** -22 * abs(x)
        assert abs(float(r.margins[j]) - x) <= dx + 1e-12
        total += ((1 - smoothing) * np.log1p(np.exp(-x)) + smoothing * np.log1p(np.exp(x))) / pairs
        slack += (dx + 2.0 ** -21) / pairs
        slope = beta / pairs * (smoothing / (1 + np.exp(-x)) - (1 - smoothing) / (1 + np.exp(x)))
        c[a:b], c[b:e] = slope, -slope
        dc[a:e] = beta / pairs * (dx / 4 + 2.0 ** -21)
    assert abs(float(r.loss) - total) <= slack + 2.0 ** -22 * total
    scored = _np(w) != 0
    assert (np.abs(_np(r.logp) - np.where(scored, logp, 0)) <= tol).all()
    c, dc = c * _np(w) * gs, dc * _np(w) * gs
    _check_grad(_np(r.grad), c, dc, np.where(scored[:, None], p, 0), _np(t).astype(np.int64), dtype)


def test_preference_rows_outside_the_answers_and_bad_starts(meq):
    z, t, w, starts, ref, _ = _pref_inputs([3, 4, 2, 2], 100, "fp32", 3)
    w.fill_(1.0)
    r = meq.preference_loss(z, t, torch.tensor([2, 5, 9], device="cuda"), ref, w, grad=True)
    g = r.grad.abs().sum(1)
    assert (g[2:9] > 0).all() and not g[:2].any() and not g[9:].any()
    for bad in ([0, 5, 4, 6, 8], [0, 3, 12, 12, 12], [-1, 2, 4, 6, 8]):  # the first pair; rows 4 .. 7 may be the second's
        r = meq.preference_loss(z, t, torch.tensor(bad, device="cuda"), ref, w, grad=True)
        m = r.margins.cpu()
        assert torch.isnan(r.loss) and torch.isnan(m[0]) and not r.grad[:4].any()


def test_margins_far_out(meq):
    """Saturated pairs: the loss is linear on one side and vanishes on the other, the gradient with it."""
    z, t, w, starts, ref, logp = _pref_inputs([2, 2, 2, 2], 50, "fp32", 3)
    w.fill_(1.0)
    ref = torch.tensor(logp, dtype=torch.float32).cuda()
    ref[:2] -= 500.0
    ref[4:6] += 500.0
    r = meq.preference_loss(z, t, starts, ref, w, beta=1.0, grad=True)
    assert abs(float(r.margins[0]) - 1000) < 0.01 and abs(float(r.margins[1]) + 1000) < 0.01
    assert abs(float(r.loss) - 500) < 0.01
    assert float(r.grad[:4].abs().max()) == 0.0 and float(r.grad[4:].abs().max()) > 1e-3


def test_masked_tokens(meq):
    """-inf and the type's lowest value as masks; a row with one token left; NaN in rows that are not scored."""
    for dtype in ("fp32", "bf16", "fp16"):
        z, t, g = _tokens(8, 1001, dtype, 2)
        lowest = torch.finfo(DT[dtype]).min
        z[0, ::2] = float("-inf")
        z[1, 1::2] = lowest
        z[2] = float("-inf")
        z[2, 5] = -3.0
        z[3] = lowest                                   # all alike
        z[4] = float("nan")
        z[5] = float("inf")
        t[0], t[1], t[2], t[3], t[4], t[5] = 1, 2, 5, 7, -100, -5
        old, adv, w, ref = _policy_inputs(z, t.clamp(min=0), g, 0.05)
        old, ref = torch.zeros(8, device="cuda"), torch.full((8,), -1.0, device="cuda")
        w = torch.full((8,), 0.125, device="cuda")
        with np.errstate(all="ignore"):
            logp, p, dist = _rows64(z, t)
        r = meq.policy_loss(z, t, old, adv, w, ref, CLIP_LOW, CLIP_HIGH, 0.05, grad=True)
        rows = [0, 1, 2, 3, 6, 7]
        got = _np(r.logp)
        assert (np.abs(got - logp)[rows] <= _tol(logp, dist)[rows]).all()
        assert got[4] == 0 and got[5] == 0 and not r.grad[4:6].any() and torch.isfinite(r.sums).all()
        _, c, size = _policy64(logp[rows], 0.0, _np(adv)[rows], 0.125, -1.0, 0.05)
        _check_grad(_np(r.grad)[rows], c, size * (2 * _tol(logp, dist)[rows] + 2.0 ** -20), p[rows], _np(t).astype(int)[rows], dtype)
        assert not r.grad[0, ::2].any() and not r.grad[1, 1::2].any()


# every way a row is taken: a warp, a CTA, a cluster, streamed (groups by row and by slot), in several rounds
ONE_TOKEN = [(7, 1, 0), (6, 9, 1), (300, 250, 0), (9, 4111, 1), (8, 32000, 0), (7, 50001, 3), (5, 151936, 0), (700, 40003, 1), (320, 100001, 0),
             (305, 151936, 0), (3, 600011, 1)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,cols,shift", ONE_TOKEN)
@pytest.mark.parametrize("mask", ["-inf", "lowest"])
def test_a_token_of_probability_one(meq, dtype, rows, cols, shift, mask):
    """One token left in each row, anywhere in it and of any size: its log-probability is 0 and its logit the row's
    log-sum-exp, exactly, in every type and way that a row is taken."""
    z = _matrix(rows, cols, dtype, 0, shift)
    z.fill_(float("-inf") if mask == "-inf" else torch.finfo(DT[dtype]).min)
    i = torch.arange(rows, device="cuda")
    t = (i * 7919 + torch.tensor([0, cols - 1, cols // 2, 5], device="cuda").repeat(rows)[:rows] * (i < 4)) % cols
    value = torch.tensor([0.0, 5.3, -7.1, 31.7, -100.3, 1000.3, 0.1, 12.9], device="cuda").repeat(rows)[:rows].to(DT[dtype])
    z[i, t] = value
    r = meq.token_logprobs(z, t)
    assert torch.equal(r.logp, torch.zeros(rows, device="cuda"))
    assert torch.equal(r.lse, value.float())
    zero, one = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    r = meq.policy_loss(z, t, zero, one, one / rows, ref_logp=zero, kl_coef=0.5)
    assert torch.equal(r.logp, zero) and float(r.sums[2]) == 0.0
    assert float(r.loss) == float(r.sums[1]) and abs(float(r.loss) + 1) <= 2.0 ** -20


# a CTA, a cluster, streamed by one CTA and by a cluster, and rows that no cluster holds: few, and streamed
@pytest.mark.parametrize("dtype,rows,cols", [("bf16", 3, 4186), ("bf16", 4, 50011), ("bf16", 700, 40110), ("bf16", 320, 100050), ("fp32", 3, 262391),
                                             ("bf16", 2, 530191), ("bf16", 130, 870657)])
def test_ratios_are_of_unrounded_log_probabilities(meq, dtype, rows, cols):
    """Rows of equal logits: logp = -log(cols), whose rounding to fp32 adds about 4.7e-7 to it. With that rounded value
    as old_logp every ratio is below 1 by as much. Allowed: 5e-8 (the correction of approximate exponentials, which are
    exact here), 9e-8 for log(cols) and its additions, two ulps of the ratio (1.2e-7), and 6e-8 for the rounded sum."""
    z, t = _matrix(rows, cols, dtype), torch.arange(rows, device="cuda")
    old = np.float32(-math.log(cols))
    ratio = math.exp(-math.log(cols) - float(old))
    assert ratio < 1 - 4.5e-7
    one = torch.ones(rows, device="cuda")
    r = meq.policy_loss(z, t, torch.full((rows,), float(old), device="cuda"), one)
    assert abs(float(r.sums[1]) / (-rows * ratio) - 1) <= 3.2e-7
    assert abs(float(r.loss) / (-rows * ratio) - 1) <= 3.2e-7


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_probable_tokens_have_no_common_bias(meq, dtype):
    """8192 tokens with p > 0.998. A sum next to 1 is rounded at most eleven times on its way, by 2^-24 each: the mean
    over the rows of eleven such errors, evenly spread, has a deviation of 1.2e-9; 1.5e-8 is twelve of them. One row
    is off by at most the eleven, and 2^-20 of the rest, which is below 2e-3."""
    rows, cols = 8192, 64
    g = torch.Generator().manual_seed(4)
    z = torch.randn(rows, cols, generator=g)
    t = torch.randint(0, cols, (rows,), generator=g)
    z[torch.arange(rows), t] = 12.0 + torch.randn(rows, generator=g)
    m = _matrix(rows, cols, dtype)
    m.copy_(z)
    logp = torch.log_softmax(m.double(), 1).gather(1, t.cuda()[:, None])[:, 0]
    sure = logp > math.log(0.998)
    assert int(sure.sum()) > 4000
    off = (meq.token_logprobs(m, t.cuda()).logp.double() - logp)[sure]
    assert float(off.abs().max()) <= 11 * 2.0 ** -24 + 2e-3 * 2.0 ** -20 and abs(float(off.mean())) <= 1.5e-8


def test_rows_without_an_answer_are_nan(meq):
    """No finite logit, +inf, NaN, a target beyond the row: that row is NaN, no other is."""
    z, t, _ = _tokens(6, 300, "fp32", 2)
    z[0] = float("-inf")
    z[1, 7] = float("inf")
    z[2, 9] = float("nan")
    t[3] = 300
    t[4] = 2 ** 40
    want, _, dist = _rows64(z[5:], t[5:])
    got = _np(meq.token_logprobs(z, t).logp)
    assert np.isnan(got[:5]).all() and abs(got[5] - want[0]) <= _tol(want, dist)[0]
    zero = torch.zeros(6, device="cuda")
    r = meq.policy_loss(z, t, zero, zero + 1, zero + 1, grad=True)
    assert torch.isnan(r.grad[:5]).any(1).all() and torch.isfinite(r.grad[5]).all() and torch.isnan(r.loss)
    # a target whose token is masked: probability zero, not NaN
    z, t, _ = _tokens(1, 300, "fp32", 2)
    z[0, t[0]] = float("-inf")
    r = meq.token_logprobs(z, t)
    assert float(r.logp[0]) == float("-inf")


@pytest.mark.parametrize("dtype,rows,cols", [("bf16", 640, 40003), ("bf16", 310, 151936), ("fp32", 310, 50001)])
def test_long_rows_without_an_answer_are_nan(meq, dtype, rows, cols):
    """The same among many long rows, and rows of the type's lowest value alone; all other rows stay as they are."""
    g = torch.Generator(device="cuda").manual_seed(cols)
    z = _matrix(rows, cols, dtype, 0, 1)
    z.copy_(torch.randn(rows, cols, generator=g, device="cuda"))
    t = torch.randint(0, cols, (rows,), generator=g, device="cuda")
    one = torch.ones(rows, device="cuda")
    clean = meq.policy_loss(z, t, -10 * one, one, grad=True)
    bad = torch.tensor([5, 70, 160, 161, 299], device="cuda")
    z[5], z[70, cols - 1], z[160, 0], z[161, cols // 2], t[299] = float("-inf"), float("inf"), float("nan"), float("nan"), cols
    z[33] = torch.finfo(DT[dtype]).min
    got = meq.token_logprobs(z, t)
    r = meq.policy_loss(z, t, -10 * one, one, grad=True)
    assert torch.equal(torch.isnan(r.logp).nonzero()[:, 0], bad) and torch.equal(torch.isnan(got.logp).nonzero()[:, 0], bad)
    assert float(got.lse[5]) == float("-inf") and bool(torch.isnan(got.lse[[70, 160, 161]]).all()) and bool(torch.isfinite(got.lse[299]))
    assert bool(torch.isnan(r.grad[bad]).any(1).all()) and bool(torch.isnan(r.sums[:2]).all())   # the loss, its surrogate part
    assert abs(float(got.logp[33]) + math.log(cols)) <= 2.0 ** -17 and abs(float(r.logp[33]) + math.log(cols)) <= 2.0 ** -17
    other = torch.ones(rows, dtype=torch.bool, device="cuda")
    other[bad], other[33] = False, False
    assert torch.equal(r.logp[other], clean.logp[other]) and torch.equal(r.grad[other], clean.grad[other])
    assert bool(torch.isfinite(r.grad[33]).all())


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_gradient_against_differences(meq, loss):
    """The change of the loss along the gradient. Step h = 1e-2: the third-order term of a symmetric
    difference is about h^2 = 1e-4 of the slope, rounding of the loss 1e-7 / h of it."""
    lengths = [5, 9, 3, 4]
    z, t, w, starts, ref, logp = _pref_inputs(lengths, 211, "fp32", 8)
    old = torch.tensor(logp + 0.05, dtype=torch.float32).cuda()
    adv = torch.linspace(0.5, 2.0, len(logp), device="cuda")  # all ratios near exp(-0.05): none near a clip edge

    def call(x, **kw):
        if loss == "policy":
            return meq.policy_loss(x, t, old, adv, w, ref, kl_coef=0.3, **kw)
        return meq.preference_loss(x, t, starts, ref, w, beta=0.5, label_smoothing=0.1, **kw)

    g = call(z, grad=True).grad
    norm = float(g.double().norm())
    v = g / norm
    h = 1e-2
    slope = (float(call(z + h * v).loss) - float(call(z - h * v).loss)) / (2 * h)
    assert abs(slope / norm - 1) < 2e-3


def test_determinism_streams_and_graphs(meq):
    z, t, w, starts, ref, logp = _pref_inputs([40, 60, 80, 20], 5003, "bf16", 8)
    old = torch.tensor(logp, dtype=torch.float32).cuda()
    adv = torch.linspace(-1, 1, len(logp), device="cuda")
    calls = [lambda **k: meq.policy_loss(z, t, old, adv, w, ref, kl_coef=0.1, grad=True, **k),
             lambda **k: meq.preference_loss(z, t, starts, ref, w, grad=True, **k),
             lambda **k: meq.token_logprobs(z, t, **k)]
    for call in calls:
        a = [x.clone() for x in call()]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        for stream in (side, side.cuda_stream):
            b = call(stream=stream)
            side.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(a, b))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c = call()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a, c))


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_a_gradient_over_saved_logits_is_noticed(meq, loss):
    """Logits that their own function keeps for its backward pass (a soft cap by tanh): written over by their gradient,
    backward raises; with the gradient elsewhere, or logits that nothing keeps, it runs."""
    n, cols = 12, 300
    t = torch.arange(n, device="cuda")
    zero, one = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda")

    def call(z, grad):
        if loss == "policy":
            return meq.policy_loss(z, t, zero - 5.0, one, one / n, grad=grad)
        return meq.preference_loss(z, t, torch.tensor([0, 5, n], device="cuda"), zero, grad=grad)

    for kept in (True, False):
        x = torch.randn(n, cols, device="cuda", requires_grad=True)
        y = torch.tanh(x) if kept else x * 2.0
        call(y.detach(), True).grad      # a new tensor: nothing is written over
        y.backward(call(y.detach(), True).grad, retain_graph=True)
        want, x.grad = x.grad, None
        z = y.detach()
        r = call(z, z)
        if kept:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                y.backward(r.grad)
        else:
            y.backward(r.grad)
            assert torch.equal(x.grad, want)
    with torch.inference_mode():         # tensors without a version counter
        z = torch.randn(n, cols, device="cuda")
        assert call(z, z).grad is z


def test_no_rows(meq):
    z = torch.zeros(0, 100, device="cuda")
    e, t = torch.zeros(0, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda")
    assert meq.token_logprobs(z, t).logp.numel() == 0
    r = meq.policy_loss(z, t, e, e, e, grad=True)
    assert not r.sums.any() and r.grad.shape == (0, 100)


def test_offsets_beyond_32_bits(meq):
    """Rows whose first elements lie past 2^31 elements and past 2^32 bytes."""
    rows, ld, cols = 5, (1 << 29) + 11, 1500
    flat = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    z = flat.view(rows, ld)[:, :cols]
    g = torch.Generator().manual_seed(1)
    z.copy_(torch.randn(rows, cols, generator=g))
    t = torch.randint(0, cols, (rows,), generator=g).cuda()
    _check_policy(meq, z, t, g, 0.05, "bf16", True)
    small = z.clone()
    assert torch.equal(meq.token_logprobs(z, t).logp, meq.token_logprobs(small, t).logp)


def test_refusals(meq):
    z, t, g = _tokens(4, 100, "fp32", 1)
    v = torch.zeros(4, device="cuda")
    for bad in (z.T, z.double(), z.cpu(), z[0], z[:, ::2], z[:1].expand(4, 100)):
        with pytest.raises(ValueError):
            meq.token_logprobs(bad, t)
    for bad in (t.int(), t[:3], t.cpu()):
        with pytest.raises(ValueError):
            meq.token_logprobs(z, bad)
    with pytest.raises(ValueError):
        meq.policy_loss(z, t, v.double(), v)
    with pytest.raises(ValueError):
        meq.policy_loss(z, t, v, v, grad=z.bfloat16())
    with pytest.raises(ValueError):
        meq.policy_loss(z, t, v, v, grad=z[:, :50])
    with pytest.raises(ValueError):
        meq.policy_loss(z, t, v, v, grad_scale=v)
    for kw in (dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_high=float("inf")), dict(kl_coef=-1.0), dict(kl_coef=0.1)):
        with pytest.raises(meq.MeqError) as e:  # the last: a KL term without ref_logp
            meq.policy_loss(z, t, v, v, **kw)
        assert e.value.status == 1 and "meq_policy_loss" in str(e.value)
    s = torch.tensor([0, 2, 4], device="cuda")
    for kw in (dict(beta=0.0), dict(beta=float("nan")), dict(label_smoothing=1.5)):
        with pytest.raises(meq.MeqError) as e:
            meq.preference_loss(z, t, s, v, **kw)
        assert e.value.status == 1 and "meq_preference_loss" in str(e.value)
    with pytest.raises(ValueError):
        meq.preference_loss(z, t, s[:2], v)
    with pytest.raises(ValueError):
        meq.preference_loss(z, t, s.int(), v)
