"""The operators of a fine-tuning step beside MeqMuon's own update, as cases that can be timed and compared.

A case is a dict of plain values. Its "call" says which operator it runs:

  adamw       one AdamW step over every parameter of a list (`meq.AdamW`): those that MeqMuon leaves
              to it (embedding, head, norm weights), or a whole model.
    layers, hidden, ffn, vocab   a Llama-style model; which: "all" its parameters, the "rest" (embedding,
              head and norm weights) or the norm "vectors" alone. layers = 0: `shapes`, "rowsxcols,..."
    bits      32: the moments in fp32; 8: in 8-bit codes with one fp32 scale per 256 elements
    param, grad   types of parameters and gradients; copy: the step also writes the parameters in bf16
    clip      the step's own gradient norm is taken first and the gradients clipped to it;
    scaled    the gradients are multiplied by a coefficient that the program already has on the device
    shift     the flat buffers start this many elements into an allocation
  logprobs    log-probabilities of the given tokens from logits (`meq.token_logprobs`)
  policy      the clipped policy loss with its KL term and the gradient of the logits (`meq.policy_loss`)
  preference  the paired preference loss and the gradient of the logits (`meq.preference_loss`)
    rows      tokens (policy, logprobs); pairs, length: pairs of answers and the mean length of one
    vocab, pad, dtype   columns of the logits, columns of padding after each row, and their type
    active    share of the tokens that are scored (the others belong to prompts or padding)
    kl        policy: the coefficient of the KL term (0: none)
"""
import math
import random

import torch

own = False

BETA1, BETA2, EPS, LR, WD, MAX_NORM, STEPS_BEFORE = 0.9, 0.95, 1e-8, 3e-4, 0.1, 1.0, 10
BLOCK = 256          # elements that share a scale in the 8-bit states; parameters start at its multiples
CLIP_LOW, CLIP_HIGH = 0.2, 0.28
PREF_BETA, SMOOTHING = 0.1, 0.05

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}


# -------------------------------------------------------------------- cases
def _adamw(layers=0, hidden=0, ffn=0, vocab=0, which="all", shapes="", bits=32, param="fp32", grad="fp32", copy=False,
           clip=False, scaled=False, shift=0, name=None):
    c = {"call": "adamw", "layers": layers, "hidden": hidden, "ffn": ffn, "vocab": vocab, "which": which, "shapes": shapes,
         "bits": bits, "param": param, "grad": grad, "copy": copy, "clip": clip, "scaled": scaled, "shift": shift}
    return c if name is None else dict(c, name=name)


def _tokens(call, rows, vocab, dtype="bf16", pad=0, active=1.0, kl=0.0, name=None):
    c = {"call": call, "rows": rows, "vocab": vocab, "pad": pad, "dtype": dtype, "active": active}
    if call == "policy":
        c["kl"] = kl
    return c if name is None else dict(c, name=name)


def _pairs(pairs, length, vocab, dtype="bf16", pad=0, active=0.7, name=None):
    c = {"call": "preference", "pairs": pairs, "length": length, "vocab": vocab, "pad": pad, "dtype": dtype, "active": active}
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # The norm weights of a 130M model, whose matrices MeqMuon steps: 25 short vectors, where launches count.
        _adamw(12, 768, 2048, 32000, "vectors", name="adamw 130m norm weights"),
        # Embedding, head and norm weights of the same model with 8-bit moments and bf16 gradients under a loss scale.
        _adamw(12, 768, 2048, 32000, "rest", bits=8, grad="bf16", scaled=True, name="adamw 130m embeddings 8-bit"),
        # Every parameter of a 350M model in mixed precision: fp32 masters, clipped fp32 gradients, a bf16 copy out.
        _adamw(24, 1024, 2736, 32000, "all", copy=True, clip=True, name="adamw 350m whole clipped"),
        # Four layers of a 1B-class model kept in bf16 alone, 8-bit moments: the least memory, an odd FFN width.
        _adamw(4, 2048, 5461, 32000, "all", bits=8, param="bf16", grad="bf16", name="adamw 1b four layers 8-bit"),
        # Scoring the candidates of one decoding step: few rows, each over the whole vocabulary.
        _tokens("logprobs", 16, 151936, name="logprobs 16 candidates"),
        # The reference model's log-probabilities of a batch of answers.
        _tokens("logprobs", 8192, 32000, active=0.8, name="logprobs 8192 tokens"),
        # One short answer in fp32: the smallest policy update.
        _tokens("policy", 24, 32000, dtype="fp32", kl=0.04, name="policy one short answer"),
        # An ordinary policy minibatch without a KL term; the vocabulary is odd, so every row starts elsewhere in its 16 bytes.
        _tokens("policy", 6000, 50001, active=0.7, kl=0.0, name="policy odd vocabulary"),
        # A large minibatch over a large vocabulary, rows padded to a multiple of 128, KL against a reference.
        _tokens("policy", 8192, 151936, pad=0, active=0.85, kl=0.02, name="policy large vocabulary"),
        # Two pairs of short answers in fp16 under a loss scale.
        _pairs(2, 40, 49152, dtype="fp16", name="preference two pairs fp16"),
        # An ordinary preference batch: 16 pairs, prompts masked.
        _pairs(16, 300, 32000, name="preference 16 pairs"),
        # A large one: long answers over a large vocabulary.
        _pairs(8, 700, 151936, active=0.8, name="preference large vocabulary"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    call = rng.choice(["adamw", "adamw", "adamw", "logprobs", "policy", "policy", "policy", "preference", "preference"])
    while True:
        if call == "adamw":
            bits = rng.choice([32, 8])
            opts = {"bits": bits, "param": rng.choice(["fp32", "fp32", "bf16"]), "grad": rng.choice(["fp32", "bf16", "bf16", "fp16"]),
                    "shift": rng.choice([0, 0, 0, 1, 3])}
            opts["copy"] = opts["param"] == "fp32" and rng.random() < 0.4
            opts["clip"] = bits == 32 and rng.random() < 0.5
            opts["scaled"] = not opts["clip"] and rng.random() < 0.4
            if rng.random() < 0.4:
                text = ",".join("%dx%d" % (_log_uniform(rng, 1, 1500), _log_uniform(rng, 1, 3000)) for _ in range(_log_uniform(rng, 1, 300)))
                c = _adamw(shapes=text, **opts)
            else:
                hidden = _log_uniform(rng, 96, 2048)
                if rng.random() < 0.6:
                    hidden = 64 * max(2, hidden // 64)
                c = _adamw(rng.randint(1, 24), hidden, int(hidden * rng.uniform(2.0, 4.0)), _log_uniform(rng, 1000, 50000),
                           rng.choice(["all", "rest", "vectors"]), **opts)
        else:
            vocab = _log_uniform(rng, 500, 160000)
            if rng.random() < 0.5:
                vocab = 64 * max(8, vocab // 64)
            opts = {"dtype": rng.choice(["bf16", "bf16", "bf16", "fp16", "fp32"]), "pad": rng.choice([0, 0, 1, 40, 128]),
                    "active": rng.choice([1.0, 0.9, 0.6, 0.3])}
            if call == "preference":
                c = _pairs(_log_uniform(rng, 1, 64), _log_uniform(rng, 2, 1000), vocab, **opts)
            else:
                if call == "policy":
                    opts["kl"] = rng.choice([0.0, 0.01, 0.1])
                c = _tokens(call, _log_uniform(rng, 1, 16000), vocab, **opts)
        if work(c)["bytes"] <= most:
            return c


# ------------------------------------------------------------------- inputs
def _shapes(case):
    """(rows, cols) of every parameter, in order."""
    if case["layers"] == 0:
        return [tuple(int(x) for x in t.split("x")) for t in case["shapes"].split(",")]
    d, f, out = case["hidden"], case["ffn"], []
    if case["which"] == "all":
        for _ in range(case["layers"]):
            out += [(d, d)] * 4 + [(f, d)] * 2 + [(d, f)]
    if case["which"] != "vectors":
        out += [(case["vocab"], d)] * 2
    return out + [(1, d)] * (2 * case["layers"] + 1)


def _offsets(shapes):
    """Element at which each parameter starts in the flat buffers, and their length."""
    at, out = 0, []
    for m, n in shapes:
        out.append(at)
        at += -(-m * n // BLOCK) * BLOCK
    return out, at


def _lengths(case):
    """Lengths of the answers, chosen and rejected in turn."""
    r, n = random.Random(case["pairs"] * 7919 + case["length"]), case["length"]
    return [max(1, int(n * r.uniform(0.5, 1.5))) for _ in range(2 * case["pairs"])]


def _rows(case):
    return sum(_lengths(case)) if case["call"] == "preference" else case["rows"]


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 29)
    return g


def _flat(size, dtype, shift):
    return torch.zeros(size + 8, dtype=dtype, device="cuda")[shift:shift + size]


def _adamw_inputs(case, seed):
    shapes, g = _shapes(case), _generator(seed)
    offsets, size = _offsets(shapes)
    used = torch.zeros(size, dtype=torch.bool, device="cuda")   # False between the parameters
    decay = torch.zeros(size, device="cuda")                    # vectors are not decayed
    s = {"shapes": shapes, "offsets": offsets, "size": size, "decay": decay, "used": used}
    scale = torch.ones(size, device="cuda")
    for i, (m, n) in enumerate(shapes):
        used[offsets[i]:offsets[i] + m * n] = True
        if m > 1:
            decay[offsets[i]:offsets[i] + m * n] = 1.0
        scale[offsets[i]:offsets[i] + m * n] = 10.0 ** (-(i % 5) / 2.0)
    # element-wise spread of the gradients over three decades, as rare tokens and outlier channels give it
    scale.mul_(torch.exp(1.5 * torch.randn(size, generator=g, device="cuda"))).mul_(1e-3).mul_(used)
    s["p"] = _flat(size, TYPES[case["param"]], case["shift"])
    s["p"].copy_(0.02 * torch.randn(size, generator=g, device="cuda") * used)
    s["g"] = _flat(size, TYPES[case["grad"]], case["shift"])
    factor = 64.0 if case["scaled"] or case["grad"] == "fp16" else 1.0
    s["g"].copy_(torch.randn(size, generator=g, device="cuda") * scale * factor)
    m = 0.3 * torch.randn(size, generator=g, device="cuda") * scale
    r = scale * (0.6 + 0.4 * torch.rand(size, generator=g, device="cuda"))
    if case["bits"] == 32:
        s["m"], s["v"] = m, r * r
    else:
        s["m_code"], s["m_scale"] = _encode(m, 127.0)
        s["r_code"], s["r_scale"] = _encode(r, 255.0)
    s["coef"] = torch.tensor([0.7 / 64.0], device="cuda") if case["scaled"] else None
    if case["copy"]:
        s["copy"] = _flat(size, torch.bfloat16, case["shift"])
    return s


def _token_inputs(case, seed):
    g, n, v = _generator(seed), _rows(case), case["vocab"]
    buf = torch.empty(n, v + case["pad"], dtype=TYPES[case["dtype"]], device="cuda")
    logits = buf[:, :v]
    step = max(1, (1 << 28) // (v + case["pad"]))
    targets = torch.randint(0, v, (n,), generator=g, device="cuda")
    boost = 2.0 + 10.0 * torch.rand(n, 1, generator=g, device="cuda")
    if case["pad"]:
        buf[:, v:] = 0.0
    logp = torch.empty(n, device="cuda")
    for i in range(0, n, step):
        z = 2.0 * torch.randn(min(step, n - i), v, generator=g, device="cuda")
        z.scatter_add_(1, targets[i:i + step, None], boost[i:i + step])
        logits[i:i + step] = z
        z = logits[i:i + step].float()
        logp[i:i + step] = z.gather(1, targets[i:i + step, None])[:, 0] - torch.logsumexp(z, 1)
    mask = torch.rand(n, generator=g, device="cuda") < case["active"]
    mask[0] = True
    targets = torch.where(mask, targets, torch.full_like(targets, -100))
    s = {"buf": buf, "logits": logits, "targets": targets}
    if case["call"] == "logprobs":
        return s
    s["weights"] = mask.float() if case["call"] == "preference" else mask.float() / mask.sum()
    s["grad"] = torch.empty(n, v + case["pad"], dtype=TYPES[case["dtype"]], device="cuda")[:, :v]
    s["scale"] = torch.tensor([4096.0 if case["dtype"] == "fp16" else 1.0], device="cuda")
    if case["call"] == "policy":
        # the policy has moved a little since it wrote the answers; no ratio lies where rounding decides whether it is clipped
        d = 0.15 * torch.randn(n, generator=g, device="cuda")
        for edge in (1.0 - CLIP_LOW, 1.0 + CLIP_HIGH):
            d = torch.where((d.exp() - edge).abs() < 1e-3, d + 4e-3, d)
        s["old_logp"] = logp - d
        s["advantages"] = 0.4 + torch.randn(n, generator=g, device="cuda")
        s["ref_logp"] = logp - 0.2 * torch.randn(n, generator=g, device="cuda") if case["kl"] else None
    else:
        lengths = _lengths(case)
        starts = [0]
        for x in lengths:
            starts.append(starts[-1] + x)
        s["starts"] = torch.tensor(starts, dtype=torch.int64, device="cuda")
        seq = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), torch.tensor(lengths, device="cuda"))
        lean = torch.where(seq % 2 == 0, 0.02, -0.01)
        s["ref_logp"] = logp - 0.1 * torch.randn(n, generator=g, device="cuda") - lean
    return s


def prepare(case, seed):
    if case["call"] != "adamw":
        return dict(_token_inputs(case, seed), case=case)
    s = dict(_adamw_inputs(case, seed), case=case)
    if own:
        from paper_2609_35701_gb300 import meq

        def views(flat):
            return [flat[o:o + m * n].view(m, n) for o, (m, n) in zip(s["offsets"], s["shapes"])]

        names = {"fp32": "float32", "bf16": "bfloat16", "fp16": "float16"}
        s["opt"] = meq.AdamW(s["shapes"], beta1=BETA1, beta2=BETA2, eps=EPS, state_bits=case["bits"],
                             param_dtype=names[case["param"]], grad_dtype=names[case["grad"]],
                             decay=[1.0 if m > 1 else 0.0 for m, _ in s["shapes"]])
        for k, t in s["opt"].state().items():
            t.copy_(s.pop(k))
        s["opt"].set_steps(STEPS_BEFORE)
        s["params"], s["grads"] = views(s["p"]), views(s["g"])
        s["copies"] = views(s["copy"]) if case["copy"] else None
        s["norm"] = torch.empty(2, device="cuda")
        if case["bits"] == 8:
            s["values"] = [torch.zeros(s["size"], device="cuda") for _ in range(2)]
    s["steps"] = STEPS_BEFORE
    return s


# ------------------------------------------------------- the 8-bit states
def _encode(x, most):
    """Codes and scales of blocks of 256: x ~ scale * (code / most)^2, with x's sign."""
    b = x.view(-1, BLOCK)
    scale = b.abs().amax(1)
    scale = torch.where(scale < 2.0 ** -126, torch.zeros_like(scale), scale)   # a reciprocal would overflow
    inv = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
    q = torch.round(most * torch.sqrt(b.abs() * inv[:, None]))
    if most > 127:  # a root above zero keeps a code above zero, since the update is divided by it
        return torch.where(b > 0, q.clamp(min=1.0), q).to(torch.uint8).view(-1), scale
    return (q * torch.sign(b)).to(torch.int8).view(-1), scale


def _decode(code, scale, most):
    t = code.float() * (1.0 / most)
    return ((t * t.abs()).view(-1, BLOCK) * scale[:, None]).view(-1)


# -------------------------------------------------------------- plain forms
def _plain_adamw(s):
    case = s["case"]
    g, p, out = s["g"].float(), s["p"].float(), {}
    if case["clip"]:
        norm = torch.sqrt((g * g).sum())
        coef = torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm))
        out["norm"] = torch.stack([norm, coef])
        g = g * coef
    elif s["coef"] is not None:
        g = g * s["coef"]
    if case["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m = _decode(s["m_code"], s["m_scale"], 127.0)
        r = _decode(s["r_code"], s["r_scale"], 255.0)
        v = r * r
    s["steps"] += 1
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * g) * (1.0 - BETA2)
    r = torch.sqrt(v)
    update = m / (r * (1.0 / math.sqrt(1.0 - BETA2 ** s["steps"])) + EPS)
    p = p * (1.0 - (LR * WD) * s["decay"]) - update * (LR / (1.0 - BETA1 ** s["steps"]))
    s["p"].copy_(p)
    out["params"] = s["p"]
    if case["copy"]:
        s["copy"].copy_(p)
        out["copy"] = s["copy"]
    if case["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        s["m_code"], s["m_scale"] = _encode(m, 127.0)
        s["r_code"], s["r_scale"] = _encode(r, 255.0)
        m = _decode(s["m_code"], s["m_scale"], 127.0)
        r = _decode(s["r_code"], s["r_scale"], 255.0)
        v = r * r
    out["m"], out["v"] = m, v
    return out


def _plain_rows(s):
    """Shifted exponentials, their sums, and the log-probability of each row's token (0 where none is scored)."""
    z = s["logits"].float()
    t = s["targets"].clamp(min=0)[:, None]
    top = z.amax(1, keepdim=True)
    zt = z.gather(1, t) - top
    e = (z - top).exp()
    total = e.sum(1, keepdim=True)
    logp = (zt - total.log())[:, 0]
    return e, total, torch.where(s["targets"] >= 0, logp, torch.zeros_like(logp)), t


def _plain_grad(s, e, total, t, c):
    """c_i (onehot - softmax) in the logits' type; zero where c is."""
    g = e.mul_(-(c[:, None] / total))
    g.scatter_add_(1, t, c[:, None])
    s["grad"].copy_(g)
    return s["grad"]


def _plain_policy(s):
    w, a, kl = s["weights"], s["advantages"], s["case"]["kl"]
    e, total, logp, t = _plain_rows(s)
    ratio = (logp - s["old_logp"]).exp()
    plain, clipped = ratio * a, ratio.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * a
    cut = plain > clipped
    surrogate = -torch.minimum(plain, clipped)
    slope = torch.where(cut, torch.zeros_like(plain), -plain)
    if kl:
        d = s["ref_logp"] - logp
        k3 = d.exp() - d - 1.0
        slope = slope + kl * (1.0 - d.exp())
    else:
        k3 = torch.zeros_like(surrogate)
    scored = w != 0
    zero = torch.zeros_like(w)
    terms = [torch.where(scored, w * x, zero) for x in (surrogate + kl * k3, surrogate, k3, cut.float())]
    c = torch.where(scored, w * slope, zero) * s["scale"]
    return {"sums": torch.stack(terms).sum(1), "logp": logp, "grad": _plain_grad(s, e, total, t, c)}


def _plain_preference(s):
    w, starts = s["weights"], s["starts"]
    e, total, logp, t = _plain_rows(s)
    n, pairs = logp.numel(), (starts.numel() - 1) // 2
    seq = torch.searchsorted(starts, torch.arange(n, device=logp.device), right=True) - 1
    d = torch.where(w != 0, w * (logp - s["ref_logp"]), torch.zeros_like(w))
    sums = torch.zeros(2 * pairs, device=logp.device).index_add_(0, seq, d).view(pairs, 2)
    margin = PREF_BETA * (sums[:, 0] - sums[:, 1])
    # -log sigma(x) = max(-x, 0) + log(1 + exp(-|x|))
    tail = torch.log1p(torch.exp(-margin.abs()))
    loss = (1.0 - SMOOTHING) * ((-margin).clamp(min=0) + tail) + SMOOTHING * (margin.clamp(min=0) + tail)
    slope = (1.0 / (1.0 + torch.exp(-margin)) - (1.0 - SMOOTHING)) * (PREF_BETA / pairs)
    c = torch.stack([slope, -slope], 1).view(-1)[seq] * w * s["scale"]
    return {"loss": loss.sum() * (1.0 / pairs), "margins": margin, "logp": logp, "grad": _plain_grad(s, e, total, t, c)}


# ------------------------------------------------------------ the operators
def _own_run(s):
    from paper_2609_35701_gb300 import meq

    case = s["case"]
    if case["call"] == "adamw":
        opt, out, coef = s["opt"], {}, s["coef"]
        if case["clip"]:
            out["norm"] = opt.grad_norm(s["grads"], max_norm=MAX_NORM, out=s["norm"])
            coef = s["norm"][1:]
        opt.step(s["params"], s["grads"], lr=LR, weight_decay=WD, grad_scale=coef, copies=s["copies"])
        out["params"] = s["p"]
        if case["copy"]:
            out["copy"] = s["copy"]
        if case["bits"] == 32:
            st = opt.state()
            out["m"], out["v"] = st["m"], st["v"]
        else:
            out["m"], out["v"] = opt.read_values(*s["values"])
        return out
    if case["call"] == "logprobs":
        return {"logp": meq.token_logprobs(s["logits"], s["targets"]).logp}
    if case["call"] == "policy":
        r = meq.policy_loss(s["logits"], s["targets"], s["old_logp"], s["advantages"], s["weights"], ref_logp=s["ref_logp"],
                            clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=case["kl"], grad=s["grad"], grad_scale=s["scale"])
        return {"sums": r.sums, "logp": r.logp, "grad": r.grad}
    r = meq.preference_loss(s["logits"], s["targets"], s["starts"], s["ref_logp"], s["weights"], beta=PREF_BETA,
                            label_smoothing=SMOOTHING, grad=s["grad"], grad_scale=s["scale"])
    return {"loss": r.loss, "margins": r.margins, "logp": r.logp, "grad": r.grad}


def run(state):
    if own:
        return _own_run(state)
    call = state["case"]["call"]
    if call == "adamw":
        return _plain_adamw(state)
    if call == "logprobs":
        return {"logp": _plain_rows(state)[2]}
    return _plain_policy(state) if call == "policy" else _plain_preference(state)


# --------------------------------------------------------------------- work
def work(case):
    if case["call"] == "adamw":
        numel = float(sum(m * n for m, n in _shapes(case)))
        moments = 16.0 if case["bits"] == 32 else 4.0 + 16.0 / BLOCK + 8.0   # 8-bit: the values returned too
        each = 2.0 * BYTES[case["param"]] + BYTES[case["grad"]] + moments + (2.0 if case["copy"] else 0.0)
        return {"bytes": each * numel, "flops": 16.0 * numel}
    rows, row = float(_rows(case)), float(case["vocab"] * BYTES[case["dtype"]])
    scored = max(1.0, rows * case["active"])
    if case["call"] == "logprobs":
        return {"bytes": scored * row + 12.0 * rows, "flops": 4.0 * scored * case["vocab"]}
    # the logits of the scored rows are read, the gradients of all are written
    return {"bytes": scored * row + rows * row + 32.0 * rows, "flops": 7.0 * scored * case["vocab"]}


# -------------------------------------------------------------------- 64 bits
def _exact_adamw(case, seed):
    s = _adamw_inputs(case, seed)
    g, p, out = s["g"].double(), s["p"].double(), {}
    if case["clip"]:
        norm = torch.linalg.vector_norm(g)
        out["norm"] = torch.stack([norm, (MAX_NORM / norm).clamp(max=1.0)])
        g = g * out["norm"][1]
    elif case["scaled"]:
        g = g * s["coef"].double()
    if case["bits"] == 32:
        m, v = s["m"].double(), s["v"].double()
    else:
        m = (s["m_scale"].double()[:, None] * (s["m_code"].double() / 127).square().view(-1, BLOCK)).view(-1) * torch.sign(s["m_code"].double())
        v = (s["r_scale"].double()[:, None] * (s["r_code"].double() / 255).square().view(-1, BLOCK)).view(-1).square()
    m = torch.lerp(g, m, BETA1)
    v = torch.lerp(g.square(), v, BETA2)
    t = STEPS_BEFORE + 1
    m_hat, v_hat = m / (1 - BETA1 ** t), v / (1 - BETA2 ** t)
    p = p - LR * WD * s["decay"].double() * p - LR * m_hat / (v_hat.sqrt() + EPS)
    out["params"] = p
    if case["copy"]:
        out["copy"] = p
    if case["bits"] == 8:
        def held(x, most):
            b = x.view(-1, BLOCK)
            top = b.abs().amax(1, keepdim=True)
            q = (most * (b.abs() / top.clamp(min=1e-300)).sqrt()).round()
            if most == 255:
                q = torch.maximum(q, (b > 0).double())
            return ((q / most).square() * top * torch.sign(b)).view(-1)

        m, v = held(m, 127), held(v.sqrt(), 255).square()
    out["m"], out["v"] = m, v
    return out


def _exact_rows(s):
    """Log-probabilities of the scored tokens, a few rows at a time in 64 bits."""
    logits, targets = s["logits"], s["targets"]
    n, v = logits.shape
    out = torch.zeros(n, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 26) // v)
    for i in range(0, n, step):
        lp = torch.log_softmax(logits[i:i + step].double(), 1)
        hit = targets[i:i + step]
        out[i:i + step] = torch.where(hit >= 0, lp.gather(1, hit.clamp(min=0)[:, None])[:, 0], out[i:i + step])
    return out


def _exact_grad(s, coefs):
    n, v = s["logits"].shape
    out = torch.zeros(n, v, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 26) // v)
    for i in range(0, n, step):
        d = -torch.softmax(s["logits"][i:i + step].double(), 1)
        at = s["targets"][i:i + step].clamp(min=0)[:, None]
        d.scatter_add_(1, at, torch.ones_like(at, dtype=torch.float64))
        out[i:i + step] = d * coefs[i:i + step, None]
    return out


def _exact_policy(case, seed):
    s = _token_inputs(case, seed)
    logp, w, a = _exact_rows(s), s["weights"].double(), s["advantages"].double()
    ratio = torch.exp(logp - s["old_logp"].double())
    bound = torch.where(a >= 0, torch.minimum(ratio, torch.full_like(ratio, 1 + CLIP_HIGH)), torch.maximum(ratio, torch.full_like(ratio, 1 - CLIP_LOW)))
    cut = (bound != ratio).double()
    k3, slope = torch.zeros_like(logp), -(1 - cut) * ratio * a
    if case["kl"]:
        x = s["ref_logp"].double() - logp
        k3 = torch.expm1(x) - x
        slope = slope - case["kl"] * torch.expm1(x)
    surrogate = -bound * a
    sums = torch.stack([(w * x).sum() for x in (surrogate + case["kl"] * k3, surrogate, k3, cut)])
    return {"sums": sums, "logp": logp, "grad": _exact_grad(s, w * slope * s["scale"].double())}


def _exact_preference(case, seed):
    s = _token_inputs(case, seed)
    logp, w = _exact_rows(s), s["weights"].double()
    d = w * (logp - s["ref_logp"].double())
    starts, pairs = s["starts"].tolist(), case["pairs"]
    coefs, margins, loss = torch.zeros_like(logp), [], 0.0
    for j in range(pairs):
        a, b, c = starts[2 * j:2 * j + 3]
        x = PREF_BETA * float(d[a:b].sum() - d[b:c].sum())
        margins.append(x)
        loss += ((1 - SMOOTHING) * math.log1p(math.exp(-x)) + SMOOTHING * math.log1p(math.exp(x))) / pairs
        slope = PREF_BETA / pairs * (SMOOTHING / (1 + math.exp(-x)) - (1 - SMOOTHING) / (1 + math.exp(x)))
        coefs[a:b], coefs[b:c] = slope, -slope
    return {"loss": torch.tensor(loss, dtype=torch.float64), "margins": torch.tensor(margins, dtype=torch.float64), "logp": logp,
            "grad": _exact_grad(s, coefs * w * s["scale"].double())}


def exact(case, seed):
    if case["call"] == "adamw":
        return _exact_adamw(case, seed)
    if case["call"] == "logprobs":
        return {"logp": _exact_rows(_token_inputs(case, seed))}
    return _exact_policy(case, seed) if case["call"] == "policy" else _exact_preference(case, seed)
