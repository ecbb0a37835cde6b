"""Embedding, norms, a loss and AdamW together, as a training step runs them, against torch in 64 bits."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U = 2.0 ** -24


@pytest.fixture(scope="module")
def meq():
    import __graft_entry__

    __graft_entry__.build()
    from paper_2609_35701_gb300 import meq as m

    return m


@pytest.fixture(scope="module")
def example(meq):
    spec = importlib.util.spec_from_file_location("finetune", os.path.join(ROOT, "examples", "finetune.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _plain(model, tokens):
    """The example's model in 64 bits with torch's own operations: fp32 logits' place taken by 64-bit ones."""
    params = [p.detach().double().requires_grad_() for p in model.hidden + model.rest]
    gate, up, down, embed, head, norm = params
    x = embed[tokens]
    h = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * norm
    x = x + (torch.nn.functional.silu(h @ gate.T) * (h @ up.T)) @ down.T
    return x @ head.T, params


def test_gradients_of_the_examples_model(example):
    """Every parameter's gradient from a given gradient of the logits. Products in fp32 (not tf32) of length L are off by
    L u of their terms' sum, which chained through the block's five products stays below 2000 u of the gradient's largest
    entries here (L <= 344, factors of order one); the bf16 logits are left out by starting from their gradient."""
    torch.backends.cuda.matmul.allow_tf32 = False
    model = example.Model(vocab=509, dim=128, ffn=344, seed=3)
    tokens = torch.randint(0, 509, (700,), generator=torch.Generator().manual_seed(1)).cuda()
    tokens[:90] = 7
    logits = model.logits(tokens)
    grad = torch.randn(700, 509, generator=torch.Generator().manual_seed(2)).cuda().bfloat16() / 64
    for p in model.hidden + model.rest:
        p.grad = None
    logits.backward(grad)
    want, params = _plain(model, tokens)
    assert float((logits.detach().double() - want.detach()).abs().max()) <= 2.0 ** -8 * float(want.detach().abs().max()) + 1e-4
    want.backward(grad.double())
    for mine, plain in zip(model.hidden + model.rest, params):
        assert float((mine.grad.double() - plain.grad).abs().max()) <= 2000 * U * float(plain.grad.abs().max())
    first = [p.grad.clone() for p in model.rest]
    for p in model.hidden + model.rest:
        p.grad = None
    example.Embedding.apply(model.rest[0], tokens).sum().backward()
    assert float(model.rest[0].grad[7, 0]) == float((tokens == 7).sum()) and first[0].shape == model.rest[0].grad.shape


def test_double_backward_is_refused(example):
    x = torch.randn(4, 8, device="cuda", requires_grad=True)
    w = torch.ones(8, device="cuda", requires_grad=True)
    (g,) = torch.autograd.grad(example.RmsNorm.apply(x, w).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_step_of_two_blocks(meq, dtype):
    """tokens -> scaled embedding -> norm -> (stand-in for a block) -> norm with the residual stream -> tied head -> policy
    loss, and back by hand, the head's gradient of the table first and the embedding's added to it; then AdamW. Against the same chain
    in 64 bits by autograd. In fp32 every step is off by a few hundred u of its terms; in bf16 each of the nine roundings
    of activations and their gradients on the way is half a step, 2^-8, of a value: 9 2^-8 of the largest entries, and the
    gradient of a softmax that is off by as much, twice that."""
    n, vocab, dim = 400, 331, 96
    t = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator().manual_seed(5)
    tokens = torch.randint(0, vocab, (n,), generator=g).cuda()
    targets = torch.randint(0, vocab, (n,), generator=g).cuda()
    tokens[::17] = -1
    targets[::17] = -1
    table = (0.3 * torch.randn(vocab, dim, generator=g)).cuda()
    w1, w2 = ((1 + 0.2 * torch.randn(dim, generator=g)).cuda() for _ in range(2))
    b1 = (0.1 * torch.randn(dim, generator=g)).cuda()
    mix = (torch.randn(dim, dim, generator=g) / dim ** 0.5).cuda()
    adv, weights = torch.randn(n, generator=g).cuda(), torch.full((n,), 1.0 / n, device="cuda")
    scale = dim ** 0.5
    torch.backends.cuda.matmul.allow_tf32 = False

    x0 = meq.embedding(tokens, table, scale=scale, dtype=t)
    a = meq.layer_norm(x0, w1, b1)
    u = (a.y.float() @ mix).to(t)
    c = meq.rms_norm(u, w2, residual=x0)
    logits = (c.y.float() @ table.T).to(t)
    old = meq.token_logprobs(logits, targets).logp
    r = meq.policy_loss(logits, targets, old, adv, weights, grad=True)
    dz = r.grad.float()
    dtable = dz.T @ c.y.float()
    dy = (dz @ table).to(t)
    gc = meq.rms_norm_grad(dy, c.h, w2, c.rstd)
    da = (gc.dx.float() @ mix.T).to(t)
    ga = meq.layer_norm_grad(da, a.h, w1, a.mean, a.rstd, dh=gc.dx)
    meq.embedding_grad(ga.dx, tokens, dtable, scale=scale, accumulate=True)

    leaves = [v.double().requires_grad_() for v in (table, w1, b1, w2)]
    e, v1, c1, v2 = leaves
    held = (tokens >= 0)[:, None]
    y0 = torch.where(held, e[tokens.clamp(min=0)] * scale, torch.zeros((), dtype=torch.float64, device="cuda"))
    z = torch.nn.functional.layer_norm(y0, (dim,), v1, c1, 1e-5) @ mix.double()
    h = y0 + z
    z = (h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-6) * v2) @ e.T
    logp = torch.log_softmax(z, 1).gather(1, targets.clamp(min=0)[:, None])[:, 0]
    ratio = torch.where(targets >= 0, (logp - logp.detach()).exp(), torch.zeros_like(logp))
    (-(ratio * adv.double() * weights.double())).sum().backward()
    limit = 4000 * U if dtype == "fp32" else 18 * 2.0 ** -8
    for name, got, leaf in (("table", dtable, e), ("w1", ga.dweight, v1), ("b1", ga.dbias, c1), ("w2", gc.dweight, v2)):
        assert float((got.double() - leaf.grad).abs().max()) <= limit * float(leaf.grad.abs().max()), name
    params, grads = [table.clone(), w1.view(1, dim).clone()], [dtable, ga.dweight.view(1, dim)]
    opt = meq.AdamW([(vocab, dim), (1, dim)], decay=[1, 0])
    norm = opt.grad_norm(grads, max_norm=1.0)
    opt.step(params, grads, lr=1e-3, grad_scale=norm[1:])
    opt.sync()
    assert np.isclose(float(norm[0]), float(torch.sqrt(dtable.double().square().sum() + ga.dweight.double().square().sum())), rtol=1e-5)
    moved = (params[0] - table).abs()
    assert float(moved.max()) <= 1.01e-3 and float(moved.max()) > 0.9e-3


def test_a_step_in_one_graph(meq):
    """The whole chain captured once and replayed on new tokens gives what the calls give."""
    n, vocab, dim = 300, 200, 64
    tokens = [_t for _t in torch.randint(0, vocab, (3, n), generator=torch.Generator().manual_seed(1)).cuda()]
    table, w = torch.randn(vocab, dim, generator=torch.Generator().manual_seed(2)).cuda(), torch.ones(dim, device="cuda")
    at, out = tokens[0].clone(), torch.empty(vocab, dim, device="cuda")

    def step(t, out):
        x = meq.embedding(t, table, scale=2.0)
        r = meq.rms_norm(x, w)
        g = meq.rms_norm_grad(r.y, x, w, r.rstd)
        meq.embedding_grad(g.dx, t, out, scale=2.0)
        return r.y, g.dweight

    step(at, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(at, out)
    for t in tokens:
        at.copy_(t)
        graph.replay()
        other = torch.empty_like(out)
        want = step(t, other)
        assert torch.equal(out, other) and all(torch.equal(p, q) for p, q in zip(held, want))


def test_other_streams_memory(meq):
    """Results of a call on a stream of its own belong to that stream: memory freed and taken again meanwhile is not theirs."""
    side = torch.cuda.Stream()
    x, w = torch.randn(2000, 512, device="cuda"), torch.ones(512, device="cuda")
    want = meq.rms_norm(x, w).y
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(side):
            y = meq.rms_norm(x, w).y
        z = meq.rms_norm(x, w, stream=side)
        torch.full((2000, 512), 7.0, device="cuda")
        side.synchronize()
        assert torch.equal(y, want) and torch.equal(z.y, want)
        del y, z


def test_calls_from_several_threads(meq):
    """Four host threads, a stream each, norms and embedding of every path and refused calls among them: the results are
    those of one thread, and a refusal's text is that of the thread's own call."""
    import threading

    shapes = [(200, 96, torch.float32), (900, 1025, torch.bfloat16), (20000, 768, torch.bfloat16), (300, 17000, torch.float16)]
    data, want = [], []

    def calls(i, stream=None):
        x, res, w, t, table, out = data[i]
        r = meq.layer_norm(x, w, w, residual=res, stream=stream)
        g = meq.layer_norm_grad(res, r.h, w, r.mean, r.rstd, dh=x, stream=stream)
        q = meq.rms_norm(x, w, stream=stream)
        p = meq.rms_norm_grad(res, x, w, q.rstd, stream=stream)
        e = meq.embedding(t, table, scale=2.0, dtype=x.dtype, stream=stream)
        meq.embedding_grad(g.dx, t, out, stream=stream)
        return list(r) + list(g) + [q.y, q.rstd] + list(p) + [e, out]

    for i, (rows, cols, dtype) in enumerate(shapes):
        g = torch.Generator().manual_seed(i)
        x, res = (torch.randn(rows, cols, generator=g).cuda().to(dtype) for _ in range(2))
        w, t = (1 + 0.1 * torch.randn(cols, generator=g)).cuda(), torch.randint(-5, 300, (rows,), generator=g).cuda()
        data.append((x, res, w, t, torch.randn(300, cols, generator=g).cuda(), torch.empty(300, cols, device="cuda")))
        want.append([v.clone() for v in calls(i)])
    torch.cuda.synchronize()
    failures, start = [], threading.Barrier(len(shapes))

    def work(i):
        try:
            stream = torch.cuda.Stream()
            start.wait()
            for _ in range(15):
                got = calls(i, stream)
                x, w = data[i][0], data[i][2]
                if i % 2:
                    with pytest.raises(meq.MeqError, match="eps"):
                        meq.rms_norm(x, w, eps=-1.0, stream=stream)
                else:
                    with pytest.raises(meq.MeqError, match="the same"):
                        meq.rms_norm(x, w, residual=x, y=data[i][1], h=data[i][1], stream=stream)
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
