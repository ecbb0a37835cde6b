"""AdamW over many tensors: against plain 64-bit arithmetic, in 32- and 8-bit states.

Tolerances. A step adds at most four roundings of 2^-24 to each term of m (two products, the two
coefficients, a sum) and six to v; m may cancel, so its bound is taken of the same recursion over
magnitudes. The parameter takes the update (about six roundings, and the
roundings of m and r: 16 * 2^-24 of the update) and two roundings of its own (2 * 2^-24 of p): taken
together 2^-20 * lr_step + 2^-22 |p|; a bf16 parameter is then rounded by half an ulp, at most 2^-8 |p| (8 significant bits). An 8-bit
value is off by at most half a code: with x = (q/Q)^2 S, |dx| <= S (2 (q/Q) (0.5/Q) + (0.5/Q)^2), and by
0.001 of a code more where fp32 decides a near-tie the other way. The one code of r that is raised to 1 is
off by up to S / Q^2.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

B1, B2, EPS = 0.9, 0.95, 1e-8
U24 = 2.0 ** -24


@pytest.fixture(scope="module")
def meq():
    import __graft_entry__

    __graft_entry__.build()
    from paper_2609_35701_gb300 import meq as m

    return m


DT = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def _make(shapes, pdt, gdt, seed, shift=0):
    """Lists of tensors that start `shift` elements into their allocations, one allocation each."""
    g = torch.Generator().manual_seed(seed)
    ps, gs = [], []
    for i, (r, c) in enumerate(shapes):
        n = r * c
        spread = torch.exp(1.5 * torch.randn(n, generator=g)) * 10.0 ** (-(i % 4)) * 1e-2
        for out, x, dt in ((ps, 0.02 * torch.randn(n, generator=g), pdt), (gs, torch.randn(n, generator=g) * spread, gdt)):
            buf = torch.zeros(n + 4, dtype=DT[dt], device="cuda")[shift:shift + n]
            buf.copy_(x)
            out.append(buf.view(r, c))
    return ps, gs


class Reference:
    """The formulas in 64 bits, entry by entry."""

    def __init__(self, n):
        self.m, self.v, self.size, self.t = [0.0] * n, [0.0] * n, [0.0] * n, 0

    def step(self, ps, gs, lr, wd, decay, scale=1.0):
        self.t += 1
        out = []
        for i, (p, g) in enumerate(zip(ps, gs)):
            g = g * scale
            self.size[i] = B1 * self.size[i] + (1 - B1) * np.abs(g)  # of the terms of m
            self.m[i] = B1 * self.m[i] + (1 - B1) * g
            self.v[i] = B2 * self.v[i] + (1 - B2) * g * g
            u = self.m[i] / (1 - B1 ** self.t) / (np.sqrt(self.v[i] / (1 - B2 ** self.t)) + EPS)
            out.append((1 - lr * wd * decay[i]) * p - lr * u)
        return out


def _np(t):
    return t.detach().cpu().double().numpy()


RAGGED = [(1, 1), (1, 255), (1, 256), (1, 257), (3, 700), (1, 2047), (1, 2048), (1, 2049), (31, 129), (64, 64)]


@pytest.mark.parametrize("pdt,gdt", [("float32", "float32"), ("float32", "bfloat16"), ("float32", "float16"),
                                     ("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("bfloat16", "float16")])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_fp32_moments_three_steps(meq, pdt, gdt, shift):
    lr, wd = 1e-3, 0.1
    decay = [float(i % 3) / 2 for i in range(len(RAGGED))]
    opt = meq.AdamW(RAGGED, param_dtype=pdt, grad_dtype=gdt, beta1=B1, beta2=B2, eps=EPS, decay=decay)
    ref = Reference(len(RAGGED))
    ps, _ = _make(RAGGED, pdt, gdt, 1, shift)
    for t in range(3):
        _, gs = _make(RAGGED, pdt, gdt, 10 + t, shift)
        before = [_np(p) for p in ps]
        opt.step(ps, gs, lr, wd)
        want = ref.step(before, [_np(g) for g in gs], lr, wd, decay)
        m, v = opt.read_values()
        for i, (r, c) in enumerate(RAGGED):
            o, n = opt.offsets[i], r * c
            got = _np(ps[i])
            tol = lr * 2 ** -18 + 2 ** -22 * np.abs(want[i]) + (2 ** -8 * np.abs(want[i]) if pdt == "bfloat16" else 0.0)
            assert (np.abs(got - want[i]) <= tol).all(), (t, i)
            mm = ref.m[i].reshape(-1)
            assert (np.abs(_np(m[o:o + n]) - mm) <= (t + 1) * 4 * U24 * ref.size[i].reshape(-1) + 1e-45).all(), (t, i)
            vv = ref.v[i].reshape(-1)
            assert (np.abs(_np(v[o:o + n]) - vv) <= (t + 1) * 6 * U24 * vv + 1e-45).all(), (t, i)
    opt.sync()
    assert opt.steps == 3
    opt.close()


def _code_bound(x, top, most):
    q = most * np.sqrt(np.abs(x) / np.where(top > 0, top, 1.0))
    half = 0.501 / most
    bound = top * (2 * (q / most) * half + half * half)
    return (np.maximum(bound, top / most ** 2) if most == 255 else bound) + 1e-45


@pytest.mark.parametrize("pdt,gdt,shift", [("float32", "float32", 0), ("float32", "bfloat16", 1), ("bfloat16", "bfloat16", 0),
                                           ("bfloat16", "float16", 3)])
def test_8bit_moments_one_step_from_values(meq, pdt, gdt, shift):
    """Each step is checked from the values that the codes before it stand for."""
    lr, wd = 1e-3, 0.1
    opt = meq.AdamW(RAGGED, param_dtype=pdt, grad_dtype=gdt, beta1=B1, beta2=B2, eps=EPS, state_bits=8)
    ps, _ = _make(RAGGED, pdt, gdt, 1, shift)
    scale = torch.tensor([0.25], device="cuda")
    for t in range(4):
        _, gs = _make(RAGGED, pdt, gdt, 20 + t, shift)
        m0, v0 = [_np(x) for x in opt.read_values()]
        before = [_np(p) for p in ps]
        opt.step(ps, gs, lr, wd, grad_scale=scale)
        m1, v1 = [_np(x) for x in opt.read_values()]
        ref = Reference(len(RAGGED))
        ref.t = t
        cut = [slice(o, o + r * c) for o, (r, c) in zip(opt.offsets, RAGGED)]
        ref.m = [m0[s].reshape(sh) for s, sh in zip(cut, RAGGED)]
        ref.v = [v0[s].reshape(sh) for s, sh in zip(cut, RAGGED)]
        ref.size = [np.abs(x) for x in ref.m]
        want = ref.step(before, [_np(g) for g in gs], lr, wd, [1.0] * len(RAGGED), 0.25)
        for i in range(len(RAGGED)):
            tol = lr * 2 ** -18 + 2 ** -22 * np.abs(want[i]) + (2 ** -8 * np.abs(want[i]) if pdt == "bfloat16" else 0.0)
            assert (np.abs(_np(ps[i]) - want[i]) <= tol).all(), (t, i)
            root = np.sqrt(ref.v[i].reshape(-1))
            for got, x, size, most in ((m1[cut[i]], ref.m[i].reshape(-1), ref.size[i].reshape(-1), 127),
                                       (np.sqrt(v1[cut[i]]), root, root, 255)):
                n = x.size
                pad = -(-n // 256) * 256
                top = np.abs(np.pad(x, (0, pad - n))).reshape(-1, 256).max(1).repeat(256)[:n]
                assert (np.abs(got - x) <= _code_bound(x, top, most) + 6 * U24 * size).all(), (t, i, most)
                if most == 255:
                    assert ((got > 0) == (x > 0)).all()
    opt.sync()
    st = opt.state()
    used = torch.zeros(st["m_code"].numel(), dtype=torch.bool, device="cuda")
    for o, (r, c) in zip(opt.offsets, RAGGED):
        used[o:o + r * c] = True
    assert not st["m_code"][~used].any() and not st["r_code"][~used].any()  # the padding stays zero
    opt.close()


def test_8bit_codes_are_those_of_the_formula(meq):
    """Codes and scales after one step from zero, against the same fp32 formula on the CPU, bit for bit."""
    shapes = [(40, 333), (1, 77)]
    opt = meq.AdamW(shapes, beta1=B1, beta2=B2, eps=EPS, state_bits=8)
    ps, gs = _make(shapes, "float32", "float32", 3)
    gs[0][0, :256] = 0.0                       # a block of zeros
    gs[1][0, 5] = 1e-15                        # far below its block: its root keeps code 1
    gs[1][0, 6] = 1e-30                        # its square is no fp32 number: its root is zero
    opt.step(ps, gs, 1e-3)
    st = {k: v.cpu() for k, v in opt.state().items()}
    for i, (r, c) in enumerate(shapes):
        n, o = r * c, opt.offsets[i]
        g = torch.zeros(-(-n // 256) * 256)
        g[:n] = gs[i].cpu().reshape(-1)
        m = g * (1.0 - B1)
        root = torch.sqrt((g * g) * (1.0 - B2))
        for x, most, code, scale in ((m, 127.0, "m_code", "m_scale"), (root, 255.0, "r_code", "r_scale")):
            b = x.view(-1, 256)
            top = b.abs().amax(1)
            inv = torch.where(top > 0, 1.0 / top, torch.zeros_like(top))
            q = torch.round(most * torch.sqrt(b.abs() * inv[:, None]))
            q = q * torch.sign(b) if most == 127.0 else torch.where(b > 0, q.clamp(min=1.0), q)
            assert torch.equal(st[scale][o // 256:o // 256 + b.shape[0]], top)
            assert torch.equal(st[code][o:o + b.numel()].float(), q.view(-1))
    assert st["r_code"][opt.offsets[1] + 5] == 1 and st["r_code"][opt.offsets[1] + 6] == 0
    opt.close()


@pytest.mark.parametrize("seed", [1, 2])
def test_8bit_codes_over_many_values(meq, seed):
    """Four million codes of each kind, over twelve orders of magnitude and three steps, bit for bit those of
    the formula in fp32, each operation rounded: no approximate root, no contracted sum decides a code."""
    n = 1 << 22
    g = torch.Generator(device="cuda").manual_seed(seed)
    opt = meq.AdamW([(1024, n // 1024)], beta1=B1, beta2=B2, eps=EPS, state_bits=8)
    size = 10.0 ** (12 * torch.rand(n // 256, generator=g, device="cuda") - 9).repeat_interleave(256)
    scale = torch.tensor([0.37], device="cuda")
    m, r = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    for _ in range(3):
        x = torch.randn(n, generator=g, device="cuda") * size * torch.exp(2.0 * torch.randn(n, generator=g, device="cuda"))
        opt.step([torch.zeros(1024, n // 1024, device="cuda")], [x.view(1024, -1)], 1e-3, grad_scale=scale)
        x = x * scale
        st, held = opt.state(), []
        m = m * B1 + x * (1.0 - B1)
        r = torch.sqrt((r * r) * B2 + (x * x) * (1.0 - B2))
        for y, most, code, scales in ((m, 127.0, "m_code", "m_scale"), (r, 255.0, "r_code", "r_scale")):
            b = y.view(-1, 256)
            top = b.abs().amax(1)
            q = torch.round(most * torch.sqrt(b.abs() * (1.0 / top)[:, None]))
            q = q * torch.sign(b) if most == 127.0 else torch.where(b > 0, q.clamp(min=1.0), q)
            assert torch.equal(st[scales], top) and torch.equal(st[code].float(), q.view(-1))
            t = q * (1.0 / most)
            held.append(((t * t.abs()) * top[:, None]).view(-1))
        m, r = held
    got_m, got_v = opt.read_values()
    assert torch.equal(got_m, m) and torch.equal(got_v, r * r)
    opt.close()


def test_copies_and_clipping(meq):
    shapes = [(50, 300), (1, 300), (7, 11)]
    opt = meq.AdamW(shapes, beta1=B1, beta2=B2, eps=EPS)
    ps, gs = _make(shapes, "float32", "float32", 5)
    copies = [torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in shapes]
    true = math.sqrt(sum(float((_np(g) ** 2).sum()) for g in gs))
    # sums of squares in fp32 over one thread's share, then double: far below 1e-6
    for max_norm in (0.5 * true, 2.0 * true, float("inf")):
        got = opt.grad_norm(gs, max_norm).cpu().numpy()
        assert abs(got[0] / true - 1) < 1e-6
        assert abs(got[1] / min(1.0, max_norm / true) - 1) < 1e-6
    out = opt.grad_norm(gs, 0.5 * true)
    before, ref = [_np(p) for p in ps], Reference(3)
    opt.step(ps, gs, 1e-3, 0.1, grad_scale=out[1:], copies=copies)
    want = ref.step(before, [_np(g) for g in gs], 1e-3, 0.1, [1.0] * 3, float(out[1]))
    for p, c, w in zip(ps, copies, want):
        assert (np.abs(_np(p) - w) <= 1e-3 * 2 ** -18 + 2 ** -22 * np.abs(w)).all()
        assert torch.equal(c, p.bfloat16())
    opt.close()


def test_norm_is_deterministic_and_takes_16_bit(meq):
    shapes = [(300, 4097)] * 3 + [(1, 3)]
    for gdt in ("bfloat16", "float16", "float32"):
        opt = meq.AdamW(shapes, grad_dtype=gdt)
        _, gs = _make(shapes, "float32", gdt, 9, 1)
        true = math.sqrt(sum(float((_np(g) ** 2).sum()) for g in gs))
        got = [opt.grad_norm(gs).clone() for _ in range(4)]
        assert abs(float(got[0][0]) / true - 1) < 1e-6
        assert all(torch.equal(got[0], x) for x in got)
        opt.close()


def test_more_entries_than_one_launch_takes(meq):
    """600 entries go in three launches; the step count moves once."""
    shapes = [(1 + i % 3, 100 + i) for i in range(600)]
    opt = meq.AdamW(shapes, beta1=B1, beta2=B2, eps=EPS)
    ref = Reference(600)
    ps, gs = _make(shapes, "float32", "float32", 2)
    for _ in range(2):
        before = [_np(p) for p in ps]
        out = opt.grad_norm(gs, 1.0)
        true = math.sqrt(sum(float((_np(g) ** 2).sum()) for g in gs))
        assert abs(float(out[0]) / true - 1) < 1e-6
        opt.step(ps, gs, 1e-3, grad_scale=out[1:])
        want = ref.step(before, [_np(g) for g in gs], 1e-3, 0.0, [1.0] * 600, float(out[1]))
        for p, w in zip(ps, want):
            assert (np.abs(_np(p) - w) <= 1e-3 * 2 ** -18 + 2 ** -22 * np.abs(w)).all()
    assert opt.steps == 2
    opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_every_block_of_a_step_reads_the_same_clock(meq, bits):
    """200 steps, one after another, of some 18000 (8 bits) or 4500 blocks: every element has the same moments and
    gradients, so any block that read the corrections of the next step would give other parameters."""
    shape = (1024, 8999)
    opt = meq.AdamW([shape], beta1=B1, beta2=B2, eps=EPS, state_bits=bits)
    p, g = torch.zeros(shape, device="cuda"), torch.full(shape, 0.5, device="cuda")
    for _ in range(200):
        opt.step([p], [g], 1e-2)
    opt.sync()
    assert opt.steps == 200 and bool((p == p[0, 0]).all())
    # m and v are exact multiples of the gradient but for their roundings: the corrected update is 1 to 2^-16 in each step
    assert abs(float(p[0, 0]) + 200 * 1e-2) <= 200 * 1e-2 * 2 ** -16 + 200 * 2.0 ** -23
    opt.close()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("before", [0, 1, 2])
def test_the_step_count_set_after_any_number_of_steps(meq, bits, before):
    """set_steps counts for the very next step whatever came before, skipped steps do not count, and 300 entries
    (two launches) move it on once."""
    shapes = [(1, 300 + i) for i in range(300)]
    kw = dict(beta1=B1, beta2=B2, eps=EPS, state_bits=bits)
    ps, gs = _make(shapes, "float32", "float32", 6)
    qs, a, b = [p.clone() for p in ps], meq.AdamW(shapes, **kw), meq.AdamW(shapes, **kw)
    scrap = [p.clone() for p in ps]
    for _ in range(before):
        a.step(scrap, gs, 1e-3)
    for v in a.state().values():
        v.zero_()
    torch.cuda.synchronize()
    nan = torch.tensor([float("nan")], device="cuda")
    for opt, x in ((a, ps), (b, qs)):
        opt.set_steps(7)
        assert opt.steps == 7
        for _ in range(3):
            opt.step(x, gs, 1e-3)
            opt.step(x, gs, 1e-3, grad_scale=nan)
        assert opt.steps == 10
    assert all(torch.equal(p, q) for p, q in zip(ps, qs))
    a.close()
    b.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_entries_do_not_depend_on_the_list(meq, bits):
    shapes = [(33, 77), (1, 5000), (128, 128)]
    kw = dict(beta1=B1, beta2=B2, eps=EPS, state_bits=bits)
    ps, gs = _make(shapes, "float32", "float32", 4)
    alone = [p.clone() for p in ps]
    whole = meq.AdamW(shapes, **kw)
    for _ in range(3):
        whole.step(ps, gs, 1e-3, 0.1)
    for i, s in enumerate(shapes):
        one = meq.AdamW([s], **kw)
        for _ in range(3):
            one.step([alone[i]], [gs[i]], 1e-3, 0.1)
        assert torch.equal(alone[i], ps[i])
        one.close()
    whole.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_checkpoint_resumes_bit_for_bit(meq, bits):
    shapes = [(33, 77), (1, 300)]
    kw = dict(beta1=B1, beta2=B2, eps=EPS, state_bits=bits)
    ps, gs = _make(shapes, "float32", "float32", 6)
    a = meq.AdamW(shapes, **kw)
    for _ in range(3):
        a.step(ps, gs, 1e-3, 0.1)
    saved = {k: v.clone() for k, v in a.state().items()}
    qs = [p.clone() for p in ps]
    b = meq.AdamW(shapes, **kw)
    for k, v in b.state().items():
        v.copy_(saved[k])
    torch.cuda.synchronize()
    b.set_steps(a.steps)
    a.step(ps, gs, 1e-3, 0.1)
    b.step(qs, gs, 1e-3, 0.1)
    for p, q in zip(ps, qs):
        # b1^t by repeated products and by pow differ by some 1e-16: the fp32 corrections are the same
        assert torch.equal(p, q)
    a.close()
    b.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_scale_that_is_not_finite_skips_the_step(meq, bits):
    shapes = [(20, 50), (1, 3)]
    opt = meq.AdamW(shapes, state_bits=bits)
    ps, gs = _make(shapes, "float32", "float32", 8)
    opt.step(ps, gs, 1e-3)
    keep = [p.clone() for p in ps] + [t.clone() for t in opt.state().values()]
    gs[1][0, 0] = float("inf")
    out = opt.grad_norm(gs, 1.0)
    assert math.isnan(float(out[1]))
    opt.step(ps, gs, 1e-3, grad_scale=out[1:])
    with pytest.raises(meq.MeqError) as e:
        opt.sync()
    assert e.value.status == 4 and "skipped" in str(e.value)
    assert all(torch.equal(a, b) for a, b in zip(keep, ps + list(opt.state().values())))
    assert opt.steps == 1
    opt.sync()  # the report cleared it
    opt.close()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_non_finite_gradient_is_reported_and_stays_in_its_block(meq, bits, value):
    shapes = [(4, 300), (4, 300)]
    opt = meq.AdamW(shapes, state_bits=bits)
    ps, gs = _make(shapes, "float32", "float32", 8)
    gs[1][1, 7] = value
    opt.step(ps, gs, 1e-3)
    with pytest.raises(meq.MeqError) as e:
        opt.sync()
    assert e.value.status == 4 and "entry 1" in str(e.value)
    assert torch.isfinite(ps[0]).all()
    m, v = opt.read_values()
    o = opt.offsets[1]
    block = slice(o + 256, o + 512) if bits == 8 else slice(o + 307, o + 308)  # element 307 of entry 1
    bad = ~(torch.isfinite(m) & torch.isfinite(v))
    assert bad[block].all()
    bad[block] = False
    assert not bad.any()
    opt.close()


def test_tiny_and_huge_moments_in_8_bits(meq):
    """Blocks whose scale is denormal are held as zero; the largest finite ones stay finite."""
    opt = meq.AdamW([(1, 512)], beta1=B1, beta2=B2, eps=EPS, state_bits=8)
    g = torch.full((1, 512), 1e-39, device="cuda")
    g[0, 256:] = 1e18
    p = torch.zeros(1, 512, device="cuda")
    opt.step([p], [g], 1e-3)
    opt.sync()
    m, v = opt.read_values()
    assert not m[:256].any() and not v[:256].any()
    assert torch.isfinite(m).all() and torch.isfinite(v).all() and (m[256:] > 0).all()
    assert torch.isfinite(p).all()
    opt.close()


def _codes(x, most):
    """Codes and scales of blocks of 256 in fp32, each operation rounded once (float32 arithmetic on the CPU)."""
    b = x.view(-1, 256)
    top = b.abs().amax(1)
    scale = torch.where(top < 2.0 ** -126, torch.zeros_like(top), top)
    inv = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
    q = torch.round(most * torch.sqrt(b.abs() * inv[:, None]))
    q = q * torch.sign(b) if most == 127.0 else torch.where(b > 0, q.clamp(min=1.0), q)
    return q.view(-1), scale


# 300 and 257 elements end in a padded block; shift 1 takes the element-by-element path
@pytest.mark.parametrize("n,shift", [(256, 0), (300, 0), (257, 0), (512, 1)])
def test_8bit_codes_of_m_of_any_size(meq, n, shift):
    """Blocks whose largest |m| lies anywhere from the least normal number up: the codes are those of the formula
    bit for bit, zeros among the elements and in the padding keep code 0."""
    tops = [1.2e-38, 1e-37, 1e-36, 4e-35, 4.7e-35, 4.8e-35, 6e-35, 1e-34, 3e-34, 1e-20, 1.0, 1e15]
    g = torch.Generator().manual_seed(n)
    for top in tops:
        x = torch.randn(n, generator=g) * torch.exp(1.5 * torch.randn(n, generator=g))
        x = x * (top / float(x.abs().max()))
        x[::7] = 0.0
        x[3], x[n - 1] = top, -top        # the largest |m| of both blocks
        opt = meq.AdamW([(1, n)], beta1=0.0, beta2=B2, eps=EPS, state_bits=8)
        grad = torch.zeros(n + 4, device="cuda")[shift:shift + n]
        grad.copy_(x)
        opt.step([torch.zeros(1, n, device="cuda")], [grad.view(1, n)], 1e-3)
        opt.sync()
        held = torch.zeros(-(-n // 256) * 256)
        held[:n] = x                      # beta1 = 0: m is the gradient
        code, scale = _codes(held, 127.0)
        st = opt.state()
        assert torch.equal(st["m_scale"].cpu(), scale), top
        assert torch.equal(st["m_code"].cpu().float(), code), top
        opt.close()


@pytest.mark.parametrize("eps", [1e-36, 1e-30, 1e-20, 1e-14, 1e-8])
@pytest.mark.parametrize("n,shift", [(512, 0), (300, 0), (256, 3)])
def test_8bit_update_with_a_small_eps(meq, eps, n, shift):
    """Gradients of 1e-19 and 3e-19 beside 1e-10 in one block: the roots of the small ones, whose squares are no
    normal fp32 numbers, still count beside any eps. An element of v is off by at most two spacings of 2^-149 beside
    its roundings, its root by half as much of itself."""
    lr = 1e-3
    opt = meq.AdamW([(1, n)], beta1=B1, beta2=B2, eps=eps, state_bits=8)
    grad, p = torch.zeros(n + 4, device="cuda")[shift:shift + n], torch.zeros(n + 4, device="cuda")[shift:shift + n]
    grad.copy_(torch.tensor([1e-10, 1e-19, -3e-19, 1e-12]).repeat(n // 4 + 1)[:n])
    opt.step([p.view(1, n)], [grad.view(1, n)], lr)
    opt.sync()
    g = _np(grad)
    v = (1 - B2) * g * g
    root = np.sqrt(v) / math.sqrt(1 - B2)
    want = -lr * g / (root + eps)
    tol = 2.0 ** -18 + 2.0 ** -149 / v * root / (root + eps)
    assert (np.abs(_np(p) - want) <= np.abs(want) * tol + 2.0 ** -149).all(), np.max(np.abs(_np(p) / want - 1))
    opt.close()


def test_8bit_codes_of_the_largest_m(meq):
    """Moments near the largest fp32 number, put into the state: a step with no gradient keeps their codes."""
    opt = meq.AdamW([(2, 256)], beta1=0.9, beta2=B2, eps=EPS, state_bits=8)
    st = opt.state()
    code = torch.randint(-127, 128, (512,), generator=torch.Generator().manual_seed(1))
    code[::5], code[0], code[256] = 0, 127, -127
    st["m_code"].copy_(code)
    st["m_scale"].copy_(torch.tensor([9.6e37, 3.4e38]))
    top = st["m_scale"].cpu() * 0.9
    torch.cuda.synchronize()
    p, z = torch.zeros(2, 256, device="cuda"), torch.zeros(2, 256, device="cuda")
    opt.step([p], [z], 1e-3)
    opt.sync()
    st = opt.state()
    assert torch.equal(st["m_code"].cpu().long(), code) and (st["m_scale"].cpu() / top - 1).abs().max() < 1e-6
    opt.close()


def test_streams_and_graph_capture(meq):
    shapes = [(100, 100), (1, 100)]
    ps, gs = _make(shapes, "float32", "float32", 8)
    qs = [p.clone() for p in ps]
    a, b = meq.AdamW(shapes), meq.AdamW(shapes)
    for _ in range(4):
        out = a.grad_norm(gs, 0.1)
        a.step(ps, gs, 1e-3, 0.1, grad_scale=out[1:])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    norm = torch.empty(2, device="cuda")
    b.grad_norm(gs, 0.1, out=norm, stream=side)
    b.step(qs, gs, 1e-3, 0.1, grad_scale=norm[1:], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.grad_norm(gs, 0.1, out=norm)
        b.step(qs, gs, 1e-3, 0.1, grad_scale=norm[1:])
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(ps, qs))
    a.close()
    b.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_host_calls_wait_for_replays_on_any_stream(meq, bits):
    """A captured step replayed on a stream that no call was made on, behind 50 ms of other work: steps, set_steps and
    sync see what the replays do."""
    shapes = [(100, 100), (1, 100)]
    ps, gs = _make(shapes, "float32", "float32", 8)
    scale = torch.ones(1, device="cuda")
    opt = meq.AdamW(shapes, state_bits=bits)
    opt.step(ps, gs, 1e-3, grad_scale=scale)
    torch.cuda.synchronize()
    graph, side, other = torch.cuda.CUDAGraph(), torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=other):
        opt.step(ps, gs, 1e-3, grad_scale=scale)

    def replays(n):
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
            for _ in range(n):
                graph.replay()

    replays(3)
    assert opt.steps == 4
    replays(2)
    opt.set_steps(10)
    torch.cuda.synchronize()
    assert opt.steps == 10
    scale.fill_(float("inf"))
    torch.cuda.synchronize()
    replays(1)
    with pytest.raises(meq.MeqError) as e:
        opt.sync()
    assert e.value.status == 4 and "skipped" in str(e.value)
    assert opt.steps == 10
    replays(1)
    opt.close()


def test_parameters_written_before_their_backward_pass_are_noticed(meq):
    """A parameter that a backward pass still to come has saved: after a step (or a copy into it) backward raises."""
    for through_copy in (False, True):
        dt = torch.bfloat16 if through_copy else torch.float32
        w = torch.randn(16, 16, device="cuda").to(dt)
        x = torch.randn(4, 16, device="cuda", dtype=dt, requires_grad=True)
        y = (x @ w).sum()
        opt = meq.AdamW([(16, 16)])
        p = torch.randn(16, 16, device="cuda") if through_copy else w
        opt.step([p], [torch.ones(16, 16, device="cuda")], 1e-3, copies=[w] if through_copy else None)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
        opt.close()


def test_8bit_training_follows_32bit(meq):
    """A noisy least-squares problem ends where 32-bit states end. The same formulas in plain arithmetic
    end 0.04 % apart; 5 % leaves room for another order of the sums."""
    losses = {}
    for bits in (32, 8):
        g = torch.Generator().manual_seed(0)
        target = torch.randn(64, 256, generator=g).cuda()
        w = torch.zeros(64, 256, device="cuda")
        opt = meq.AdamW([(64, 256)], beta1=B1, beta2=B2, eps=EPS, state_bits=bits)
        tail = []
        for t in range(600):
            x = torch.randn(32, 64, generator=g).cuda()
            e = x @ (w - target) + torch.randn(32, 256, generator=g).cuda()
            opt.step([w], [(x.T @ e / 32).contiguous()], 1e-2)
            if t >= 500:
                tail.append(float((w - target).square().mean()))
        losses[bits] = np.mean(tail)
        opt.close()
    assert losses[32] < 2e-3 and abs(losses[8] / losses[32] - 1) < 0.05, losses


def test_refusals(meq):
    for kw in (dict(state_bits=16), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0)):
        with pytest.raises(meq.MeqError) as e:
            meq.AdamW([(4, 4)], **kw)
        assert e.value.status == 1
    with pytest.raises(meq.MeqError):
        meq.AdamW([(4, 4)], param_dtype="float16")
    with pytest.raises(meq.MeqError):
        meq.AdamW([(4, 4)], decay=[float("nan")])
    opt = meq.AdamW([(4, 4), (1, 3)])
    ps, gs = _make([(4, 4), (1, 3)], "float32", "float32", 1)
    for bad_p, bad_g in ((ps[:1], gs), (ps, [gs[0].bfloat16(), gs[1]]), ([ps[0].T, ps[1]], gs), ([ps[0].cpu(), ps[1]], gs),
                         (ps, [gs[0][:2], gs[1]])):
        with pytest.raises(ValueError):
            opt.step(bad_p, bad_g, 1e-3)
    with pytest.raises(ValueError):
        opt.step(ps, gs, 1e-3, grad_scale=torch.ones(2, device="cuda"))
    with pytest.raises(ValueError):
        opt.step(ps, gs, 1e-3, copies=ps)
    with pytest.raises(meq.MeqError):
        opt.step(ps, gs, float("nan"))
    with pytest.raises(meq.MeqError):
        opt.grad_norm(gs, 0.0)
    with pytest.raises(meq.MeqError):
        opt.set_steps(-1)
    before = [p.clone() for p in ps]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, ps)) and opt.steps == 0
    opt.close()
