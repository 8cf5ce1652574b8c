"""Operators for policies over token vocabularies, as cases that can be timed: the log-probability of the taken token, the clipped
policy loss with a KL term, the preference loss over pairs of answers, and activation checkpoints in 8 bits with their use in the
backward pass.  Each has a plain form in elementary torch operations; with `own` the framework's entry points are called instead
(paper_2104_06272_b200.tokens).

A case is a dict of plain values.  `kind` says which operator it passes through:

  logp        log-probability and entropy of the taken tokens; with back=True the gradient of the logits too
  policy      the clipped loss from log-probabilities: statistics, gradients of the log-probabilities and entropies
  policy_grad the clipped loss from logits: statistics, log-probabilities, entropies and the gradient of the logits
  pairs       the preference loss from log-probabilities: statistics, margins, gradient of the log-probabilities
  pairs_grad  the same from logits: log-probabilities, loss, gradient of the logits
  ckpt        an activation function whose input is kept in 8 bits, and the gradient of that input from what was kept
  wgrad       gradient of a layer's weights from its checkpointed input and the gradient of its output

Rows of the logits are the tokens of all sequences, one sequence after the other (`offsets`); `behind` rows belong to no
sequence (the padding of a packed batch), `ignored` is the share of prompt tokens, which carry no loss.
"""
from __future__ import annotations

import math

import torch

own = False

F32, BF16, F16 = "float32", "bfloat16", "float16"
FIELDS = {
    "logp": dict(dtype=BF16, back=True, pad=0, ignored=0.0, banned=False, scale=1.0),
    "policy": dict(seqs=1, mean="token", kl="k3", behind=0, ignored=0.1, dual=0.0),
    "policy_grad": dict(dtype=BF16, seqs=1, mean="token", kl="k3", behind=0, ignored=0.1, pad=0, banned=False, dual=0.0, scale=1.0),
    "pairs": dict(loss="sigmoid", mean=False, behind=0, ignored=0.2),
    "pairs_grad": dict(dtype=BF16, loss="sigmoid", mean=False, behind=0, ignored=0.2, pad=0),
    "ckpt": dict(dtype=BF16, act="relu", pad=0),
    "wgrad": dict(dtype=BF16, act="relu", pad=0),
}


def _case(name, kind, **more):
    return {"name": name, "kind": kind, **FIELDS[kind], **more}


def listed():
    return [
        # One generation step scored for 64 streams: few rows, a long vocabulary, nothing to differentiate.
        _case("logp_step", "logp", R=64, V=32000, back=False),
        # The framework's own four actions at its largest batch of environments, gradient included.
        _case("logp_actions", "logp", R=131072, V=4, dtype=F32),
        # A training batch over a vocabulary of odd size: no row but the first starts on a vector's boundary.
        _case("logp_train", "logp", R=4096, V=50021, dtype=F16, ignored=0.3, banned=True, scale=0.8),
        # A small group of answers whose log-probabilities are already there: the time is that of the launches.
        _case("policy_tokens", "policy", R=1000, seqs=16, mean="sequence", behind=24),
        # A full update: 8192 tokens of 32 answers over a vocabulary of 131072.
        _case("policy_grad", "policy_grad", R=8192, V=131072, seqs=32, behind=61),
        # Preference pairs from stored log-probabilities, answers from nothing to a few thousand tokens.
        _case("pairs", "pairs", R=262144, P=256, behind=100),
        # The same from logits, few long answers, an odd vocabulary.
        _case("pairs_grad", "pairs_grad", R=4099, V=32003, P=8, loss="squared", mean=True),
        # One layer of the smallest workload (64 environments, 64 units).
        _case("ckpt_small", "ckpt", R=64, K=64, dtype=F32),
        # The widest workload's recorded rows (16384 environments, 32 steps, 1024 units).
        _case("ckpt_large", "ckpt", R=524288, K=1024, act="silu"),
        # Second-layer gradient of the smallest workload: 64 environments, 16 steps, 64 units, full precision.
        _case("wgrad_small", "wgrad", R=1024, K=64, N=64, dtype=F32),
        # Odd sizes throughout.
        _case("wgrad_odd", "wgrad", R=5003, K=777, N=4099, act="identity"),
        # Second-layer gradient of the widest workload.
        _case("wgrad_large", "wgrad", R=524288, K=1024, N=1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("logp", "logp", "policy", "policy_grad", "policy_grad", "pairs", "pairs_grad", "ckpt", "ckpt", "wgrad", "wgrad"))
    c = {"kind": kind, **FIELDS[kind]}
    dtype = rng.choice((BF16, BF16, F32, F16))
    pad = rng.choice((0, 0, 1, 8, 24))
    if kind in ("logp", "policy_grad", "pairs_grad"):
        V = _log(rng, 2, 200000)
        R = min(_log(rng, 1, 131072), max(1, 500_000_000 // V))
        c.update(R=R, V=V, dtype=dtype, pad=pad)
    if kind == "logp":
        c.update(back=rng.random() < 0.7, ignored=rng.choice((0.0, 0.4)), banned=c["V"] > 64 and rng.random() < 0.5, scale=rng.choice((1.0, 1.0, 0.7, 1.3)))
    elif kind in ("policy", "policy_grad"):
        if kind == "policy":
            c["R"] = _log(rng, 1, 1 << 20)
        else:
            c.update(banned=c["V"] > 64 and rng.random() < 0.5, scale=rng.choice((1.0, 1.0, 0.7)))
        c.update(seqs=min(c["R"], _log(rng, 1, 2048)), mean=rng.choice(("token", "sequence", "fixed")), kl=rng.choice(("none", "k1", "k2", "k3", "k3")),
                 behind=rng.randint(0, c["R"] // 8), ignored=rng.choice((0.0, 0.3)), dual=rng.choice((0.0, 0.0, 3.0)))
    elif kind in ("pairs", "pairs_grad"):
        if kind == "pairs":
            c["R"] = _log(rng, 4, 1 << 20)
        c["R"] = max(4, c["R"])
        c.update(P=max(1, min(c["R"] // 4, _log(rng, 1, 1024))), loss=rng.choice(("sigmoid", "hinge", "squared")), mean=rng.random() < 0.4,
                 behind=rng.randint(0, c["R"] // 8), ignored=rng.choice((0.0, 0.3)))
    elif kind == "ckpt":
        K = _log(rng, 1, 16384)
        c.update(K=K, R=min(_log(rng, 1, 524288), 200_000_000 // K), dtype=dtype, pad=pad, act=rng.choice(("identity", "relu", "silu", "gelu")))
    else:
        K, N = _log(rng, 1, 4096), _log(rng, 1, 32768)
        R = _log(rng, 1, 524288)
        R = max(1, min(R, int(4e11 / (2.0 * K * N)), 400_000_000 // max(K, N)))
        c.update(K=K, N=N, R=R, dtype=dtype, pad=pad, act=rng.choice(("identity", "relu")))
    return c


# ---------------------------------------------------------------------------------------------------------------------
# inputs

CLIP_LOW, CLIP_HIGH, KL_COEF, ENTROPY_COEF = 0.2, 0.28, 0.05, 0.01
BETA, MARGIN, SMOOTHING = 0.1, 0.05, 0.1
BLOCK, E_MIN, E_MAX = 32, -117, 120  # a checkpoint's block of columns; exponents of its scales


def _dtype(case):
    return getattr(torch, case["dtype"])


def _logits(case, tokens, gen):
    """Spread-out scores with the taken token among the likely ones, as it is when it was sampled; a banned token (one that the
    sampler may not take) has no probability."""
    R, V, dtype = case["R"], case["V"], _dtype(case)
    out = torch.empty(R, V + case["pad"], dtype=dtype, device="cuda")
    step = max(1, (1 << 26) // V)
    for r in range(0, R, step):
        n = min(step, R - r)
        x = torch.randn(n, V, generator=gen, device="cuda") * 2.5
        t = tokens[r: r + n].clamp(min=0)
        if case.get("banned"):
            x[:, torch.arange(V, device="cuda") % 16 == 5] = float("-inf")
        x[torch.arange(n, device="cuda"), t] = torch.randn(n, generator=gen, device="cuda") + 5.0
        out[r: r + n, :V] = x.to(dtype)
    out[:, V:] = float("nan")  # between the rows lies something else
    return out[:, :V]


def _tokens(case, gen):
    R, V = case["R"], case["V"]
    tokens = torch.randint(0, V, (R,), generator=gen, device="cuda")
    share = case.get("ignored", 0.0)
    if share:
        tokens[torch.rand(R, generator=gen, device="cuda") < share] = -100
    return tokens


def _offsets(rows, seqs, gen):
    cuts = torch.randint(0, rows + 1, (seqs - 1,), generator=gen, device="cuda").sort().values
    ends = torch.tensor([0, rows], device="cuda")
    return torch.cat((ends[:1], cuts, ends[1:]))


def _logp_of(logits, tokens, scale):
    """Of the inputs, a few rows at a time."""
    out, step = [], max(1, (1 << 26) // logits.shape[1])
    for r in range(0, logits.shape[0], step):
        x = logits[r: r + step].double() * scale
        t = tokens[r: r + step].clamp(min=0)
        out.append((x.gather(1, t[:, None])[:, 0] - x.logsumexp(1)).float())
    return torch.cat(out)


def _policy_inputs(s, case, logp, gen):
    """What the policy that sampled the tokens, and a reference policy, gave them; one advantage for each answer."""
    R = case["R"]
    rows = R - case["behind"]
    noise = lambda sd: torch.randn(R, generator=gen, device="cuda") * sd  # noqa: E731
    old = logp + noise(0.15)
    # a ratio within rounding of the clip's edge would be a decision, not a number: such a row is moved off it
    ratio = torch.exp((logp - old).double())
    for edge in (1.0 - CLIP_LOW, 1.0 + CLIP_HIGH, case["dual"] or 1.0 + CLIP_HIGH):
        old = torch.where((ratio / edge - 1.0).abs() < 1e-4, old + 2e-3, old)
    s["old"], s["ref"] = old, (logp + noise(0.3)) if case["kl"] != "none" else None
    s["offsets"] = _offsets(rows, case["seqs"], gen)
    seq = torch.searchsorted(s["offsets"], torch.arange(R, device="cuda"), right=True) - 1
    s["adv"] = torch.randn(case["seqs"], generator=gen, device="cuda")[seq.clamp(0, case["seqs"] - 1)].contiguous()
    s["divisor"] = 0.5 * R


def _codes(x):
    """A checkpoint as it lies in memory: codes uint8 [R][K rounded up to 32], scales uint8 [R][blocks]."""
    R, K = x.shape
    Kp = (K + BLOCK - 1) // BLOCK * BLOCK
    codes = torch.zeros(R, Kp, dtype=torch.uint8, device="cuda")
    scales = torch.empty(R, Kp // BLOCK, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // Kp)
    for r in range(0, R, step):
        v = torch.zeros(min(step, R - r), Kp, device="cuda")
        v[:, :K] = x[r: r + step].float()
        v = v.view(v.shape[0], -1, BLOCK)
        E = _exponent(v.abs().amax(2))
        scales[r: r + step] = (E + 127).to(torch.uint8)
        codes[r: r + step] = torch.ldexp(v, -E[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(v.shape[0], Kp)
    return codes, scales


def _exponent(amax):
    """The smallest power of two that brings a block's largest value within the 448 of an e4m3 number."""
    f, e = torch.frexp(amax)
    E = torch.where(f > 0.875, e - 8, e - 9)
    return torch.where(amax > 0, E, E_MIN).clamp(E_MIN, E_MAX)


def _matrix(R, C, pad, dtype, gen, sd=1.0):
    """Activations differ in size from unit to unit."""
    out = torch.empty(R, C + pad, dtype=dtype, device="cuda")
    size = torch.exp(torch.randn(C, generator=gen, device="cuda") * 0.5) * sd
    step = max(1, (1 << 27) // C)
    for r in range(0, R, step):
        n = min(step, R - r)
        out[r: r + n, :C] = (torch.randn(n, C, generator=gen, device="cuda") * size).to(dtype)
    out[:, C:] = float("nan")
    return out[:, :C]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 7)
    kind, s = case["kind"], {"case": case}
    if kind in ("logp", "policy_grad", "pairs_grad"):
        s["tokens"] = _tokens(case, gen)
        s["logits"] = _logits(case, s["tokens"], gen)
    if kind == "logp":
        s["dlogp"] = torch.randn(case["R"], generator=gen, device="cuda") / case["R"]
        s["dentropy"] = torch.full((case["R"],), -ENTROPY_COEF / case["R"], device="cuda")
    elif kind == "policy":
        s["logp"] = -torch.rand(case["R"], generator=gen, device="cuda").add(1e-3).log().abs()
        s["entropy"] = torch.rand(case["R"], generator=gen, device="cuda") * 4.0
        s["mask"] = torch.rand(case["R"], generator=gen, device="cuda") >= case["ignored"]
        _policy_inputs(s, case, s["logp"], gen)
    elif kind == "policy_grad":
        _policy_inputs(s, case, _logp_of(s["logits"], s["tokens"], case["scale"]), gen)
    elif kind in ("pairs", "pairs_grad"):
        R = case["R"]
        if kind == "pairs":
            s["logp"] = -torch.rand(R, generator=gen, device="cuda").add(1e-3).log().abs()
            s["mask"] = torch.rand(R, generator=gen, device="cuda") >= case["ignored"]
            at = s["logp"]
        else:
            at = _logp_of(s["logits"], s["tokens"], 1.0)
        s["ref"] = at + 0.1 * torch.randn(R, generator=gen, device="cuda")
        s["offsets"] = _offsets(R - case["behind"], 2 * case["P"], gen)
    elif kind == "ckpt":
        s["x"] = _matrix(case["R"], case["K"], case["pad"], _dtype(case), gen)
        s["dy"] = _matrix(case["R"], case["K"], 0, _dtype(case), gen, 1e-3)
    else:
        x = _matrix(case["R"], case["K"], 0, torch.bfloat16, gen)
        s["codes"], s["scales"] = _codes(x)
        s["dy"] = _matrix(case["R"], case["N"], case["pad"], _dtype(case), gen, 1e-2)
    if own:
        from paper_2104_06272_b200 import tokens as tk

        if kind in ("policy", "policy_grad"):
            s["objective"] = tk.policy_objective(clip_low=CLIP_LOW, clip_high=CLIP_HIGH, dual_clip=case["dual"], kl=case["kl"], kl_coef=KL_COEF,
                                                 entropy_coef=ENTROPY_COEF, mean=case["mean"], divisor=s["divisor"])
        elif kind in ("pairs", "pairs_grad"):
            s["objective"] = tk.preference_objective(case["loss"], beta=BETA, margin=MARGIN, smoothing=SMOOTHING, mean=case["mean"])
        elif kind == "wgrad":
            s["ckpt"] = tk.Checkpoint(s["codes"], s["scales"], case["K"])
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2104_06272_b200 import tokens as tk

    case = s["case"]
    kind = case["kind"]
    if kind == "logp":
        o = tk.logp(s["logits"], s["tokens"], scale=case["scale"])
        out = {"logp": o.logp, "entropy": o.entropy}
        if case["back"]:
            out["dlogits"] = tk.logp_backward(s["logits"], s["tokens"], o.norm, s["dlogp"], entropy=o.entropy, dentropy=s["dentropy"], scale=case["scale"])
        return out
    if kind == "policy":
        o = tk.policy_loss(s["objective"], s["logp"], s["old"], s["adv"], ref_logp=s["ref"], entropy=s["entropy"], mask=s["mask"], offsets=s["offsets"])
        return {"stats": o.stats, "dlogp": o.dlogp, "dentropy": o.dentropy}
    if kind == "policy_grad":
        o = tk.policy_grad(s["objective"], s["logits"], s["tokens"], s["old"], s["adv"], ref_logp=s["ref"], offsets=s["offsets"], scale=case["scale"])
        return {"stats": o.stats, "logp": o.logp, "entropy": o.entropy, "dlogits": o.dlogits}
    if kind == "pairs":
        o = tk.preference_loss(s["objective"], s["logp"], s["offsets"], ref_logp=s["ref"], mask=s["mask"])
        return {"stats": o.stats, "margin": o.margin, "dlogp": o.dlogp}
    if kind == "pairs_grad":
        p = tk.logp(s["logits"], s["tokens"], entropy=False)
        o = tk.preference_loss(s["objective"], p.logp, s["offsets"], ref_logp=s["ref"], tokens=s["tokens"])
        return {"stats": o.stats, "margin": o.margin, "dlogits": tk.logp_backward(s["logits"], s["tokens"], p.norm, o.dlogp)}
    if kind == "ckpt":
        y, ck = tk.ckpt_forward(s["x"], case["act"])
        return {"y": y, "kept": tk.ckpt_unpack(ck, s["x"].dtype), "dx": tk.ckpt_backward(ck, s["dy"], case["act"])}
    return {"dw": tk.ckpt_weight_grad(s["ckpt"], s["dy"], case["act"])}


def _plain_logp(logits, tokens, scale):
    """Log-probabilities of all tokens and, of the counted rows, those of the taken ones and the entropies."""
    counted = tokens >= 0
    x = logits.float() * scale
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    all_logp = x - top - torch.log(e.sum(1, keepdim=True))
    p = torch.exp(all_logp)
    entropy = -(p * all_logp.clamp(min=-1e30)).sum(1)
    logp = all_logp.gather(1, tokens.clamp(min=0)[:, None])[:, 0]
    zero = torch.zeros_like(logp)
    return all_logp, p, torch.where(counted, logp, zero), torch.where(counted, entropy, zero)


def _plain_dlogits(all_logp, p, tokens, entropy, dlogp, dentropy, scale, dtype):
    counted = tokens >= 0
    g = -dlogp[:, None] * p
    g.scatter_add_(1, tokens.clamp(min=0)[:, None], dlogp[:, None])
    if dentropy is not None:
        g -= dentropy[:, None] * p * (all_logp.clamp(min=-1e30) + entropy[:, None])
    return torch.where(counted[:, None], g * scale, torch.zeros_like(g)).to(dtype)


def _plain_policy(s, case, logp, entropy, counted):
    R = case["R"]
    seq = torch.searchsorted(s["offsets"], torch.arange(R, device="cuda"), right=True) - 1
    counted = counted & (seq >= 0) & (seq < case["seqs"])
    n = torch.zeros(case["seqs"], device="cuda").index_add_(0, seq.clamp(0, case["seqs"] - 1), counted.float())
    if case["mean"] == "token":
        w = counted.float() / n.sum().clamp(min=1)
    elif case["mean"] == "sequence":
        w = counted.float() / (n[seq.clamp(0, case["seqs"] - 1)].clamp(min=1) * (n > 0).sum().clamp(min=1))
    else:
        w = counted.float() / s["divisor"]
    d = logp - s["old"]
    A = s["adv"]
    r = torch.exp(d)
    inside = ~(((A > 0) & (r > 1 + CLIP_HIGH)) | ((A < 0) & (r < 1 - CLIP_LOW)))
    pg = torch.maximum(-r * A, -r.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * A)
    if case["dual"]:
        pg = torch.where(A < 0, torch.minimum(pg, -case["dual"] * A), pg)
        inside = inside & ~((A < 0) & (r > case["dual"]))
    dlogp = torch.where(inside, -r * A, torch.zeros_like(r))
    kl = torch.zeros_like(d)
    if case["kl"] != "none":
        z = (logp - s["ref"]).double()  # exp(-z) - 1 + z is lost in 32 bits for small z
        if case["kl"] == "k1":
            kl, dkl = z, torch.ones_like(z)
        elif case["kl"] == "k2":
            kl, dkl = z * z / 2, z
        else:
            kl, dkl = torch.exp(-z) - 1 + z, 1 - torch.exp(-z)
        kl, dlogp = kl.float(), dlogp + KL_COEF * dkl.float()
    # (a row that does not count may hold anything)
    total = lambda v: torch.where(counted, w * v, torch.zeros_like(w)).double().sum()  # noqa: E731
    terms = [total(pg), total(kl), total(entropy), total((~inside).float()), total(-d)]
    loss = terms[0] + KL_COEF * terms[1] - ENTROPY_COEF * terms[2]
    return torch.stack([loss] + terms).float(), torch.where(counted, w * dlogp, torch.zeros_like(w)), -ENTROPY_COEF * w


def _plain_pairs(s, case, logp, counted):
    R, P = case["R"], case["P"]
    seq = torch.searchsorted(s["offsets"], torch.arange(R, device="cuda"), right=True) - 1
    counted = counted & (seq >= 0) & (seq < 2 * P)
    at = seq.clamp(0, 2 * P - 1)
    n = torch.zeros(2 * P, device="cuda").index_add_(0, at, counted.float())
    zero = torch.zeros_like(logp)
    # (sums of thousands of log-probabilities, of which the difference counts)
    a = torch.zeros(2 * P, dtype=torch.float64, device="cuda").index_add_(0, at, torch.where(counted, logp - s["ref"], zero).double())
    if case["mean"]:
        a = a / n.clamp(min=1)
    there = (n[:P] > 0) & (n[P:] > 0)
    z = BETA * (a[:P] - a[P:]) - MARGIN
    sp = lambda v: torch.clamp(v, min=0) + torch.log1p(torch.exp(-v.abs()))  # noqa: E731
    if case["loss"] == "sigmoid":
        loss = (1 - SMOOTHING) * sp(-z) + SMOOTHING * sp(z)
        dz = -(1 - SMOOTHING) / (1 + torch.exp(z)) + SMOOTHING / (1 + torch.exp(-z))
    elif case["loss"] == "hinge":
        loss, dz = torch.clamp(1 - z, min=0), -(z < 1).double()
    else:
        loss, dz = ((z - 0.5) / BETA) ** 2, 2 * (z - 0.5) / BETA ** 2
    pairs = there.double().sum().clamp(min=1)
    mean = lambda v: torch.where(there, v, torch.zeros_like(v)).sum() / pairs  # noqa: E731
    stats = torch.stack([mean(loss), mean((z > 0).double()), mean(BETA * a[:P]), mean(BETA * a[P:]), mean(z)]).float()
    ds = torch.where(there, BETA * dz / pairs, torch.zeros_like(dz))
    ds = torch.cat((ds, -ds))
    if case["mean"]:
        ds = ds / n.clamp(min=1)
    return stats, torch.where(there, z, torch.zeros_like(z)).float(), torch.where(counted, ds.float()[at], zero)


def _plain_act(act, x):
    if act == "relu":
        return x.clamp(min=0), (x > 0).float()
    if act == "silu":
        g = 1 / (1 + torch.exp(-x))
        return x * g, g * (1 + x * (1 - g))
    if act == "gelu":
        c = 0.5 * (1 + torch.erf(x * math.sqrt(0.5)))
        return x * c, c + x * torch.exp(-0.5 * x * x) * (1 / math.sqrt(2 * math.pi))
    return x, torch.ones_like(x)


def _plain_kept(x):
    """What a checkpoint gives back: every block of 32 columns as e4m3 numbers (3 bits of fraction, exponents from -6 on) times a
    power of two; ties to even."""
    R, K = x.shape
    v = torch.zeros(R, (K + BLOCK - 1) // BLOCK * BLOCK, device="cuda")
    v[:, :K] = x.float()
    v = v.view(R, -1, BLOCK)
    E = _exponent(v.abs().amax(2))[:, :, None]
    q = torch.ldexp(v, -E)
    step = (torch.frexp(q)[1] - 1).clamp(min=-6) - 3
    q = torch.ldexp(torch.round(torch.ldexp(q, -step)), step)
    return torch.ldexp(q, E).view(R, -1)[:, :K]


def _plain_values(codes, scales, K):
    v = codes.view(torch.float8_e4m3fn).float().view(codes.shape[0], -1, BLOCK)
    return torch.ldexp(v, scales.int()[:, :, None] - 127).view(codes.shape[0], -1)[:, :K]


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind in ("logp", "policy_grad", "pairs_grad"):
        scale = case.get("scale", 1.0)
        all_logp, p, logp, entropy = _plain_logp(s["logits"], s["tokens"], scale)
        counted = s["tokens"] >= 0
    if kind == "logp":
        out = {"logp": logp, "entropy": entropy}
        if case["back"]:
            out["dlogits"] = _plain_dlogits(all_logp, p, s["tokens"], entropy, s["dlogp"], s["dentropy"], scale, s["logits"].dtype)
        return out
    if kind == "policy":
        stats, dlogp, dentropy = _plain_policy(s, case, s["logp"], s["entropy"], s["mask"])
        return {"stats": stats, "dlogp": dlogp, "dentropy": dentropy}
    if kind == "policy_grad":
        stats, dlogp, dentropy = _plain_policy(s, case, logp, entropy, counted)
        return {"stats": stats, "logp": logp, "entropy": entropy,
                "dlogits": _plain_dlogits(all_logp, p, s["tokens"], entropy, dlogp, dentropy, scale, s["logits"].dtype)}
    if kind == "pairs":
        stats, margin, dlogp = _plain_pairs(s, case, s["logp"], s["mask"])
        return {"stats": stats, "margin": margin, "dlogp": dlogp}
    if kind == "pairs_grad":
        stats, margin, dlogp = _plain_pairs(s, case, logp, counted)
        return {"stats": stats, "margin": margin, "dlogits": _plain_dlogits(all_logp, p, s["tokens"], None, dlogp, None, 1.0, s["logits"].dtype)}
    if kind == "ckpt":
        dtype, kept = s["x"].dtype, _plain_kept(s["x"])
        y = _plain_act(case["act"], s["x"].float())[0].to(dtype)
        return {"y": y, "kept": kept.clamp(-torch.finfo(dtype).max, torch.finfo(dtype).max).to(dtype),
                "dx": (s["dy"].float() * _plain_act(case["act"], kept)[1]).to(dtype)}
    dw = torch.zeros(case["K"], case["N"], dtype=torch.float64, device="cuda")
    for r in range(0, case["R"], 8192):  # (sums over many thousand rows in 64 bits)
        x = _plain_values(s["codes"][r: r + 8192], s["scales"][r: r + 8192], case["K"])
        dw += _plain_act(case["act"], x)[0].t() @ s["dy"][r: r + 8192].float()
    return {"dw": dw.float()}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("logp", "policy_grad", "pairs_grad"):
        return _exact_logits(s, case)
    if kind == "policy":
        st, g, h = _exact_policy(s, case, s["logp"].double(), s["entropy"].double(), s["mask"])
        return {"stats": st, "dlogp": g, "dentropy": h}
    if kind == "pairs":
        st, z, g = _exact_pairs(s, case, s["logp"].double(), s["mask"])
        return {"stats": st, "margin": z, "dlogp": g}
    if kind == "ckpt":
        return _exact_ckpt(s, case)
    table = _exact_table()
    dw = torch.zeros(case["K"], case["N"], dtype=torch.float64, device="cuda")
    for r in range(0, case["R"], 32768):
        c = s["codes"][r: r + 32768].long()
        x = table[c] * torch.exp2(s["scales"][r: r + 32768].double() - 127).repeat_interleave(BLOCK, 1)
        x = x[:, : case["K"]]
        dw += (x * (x > 0) if case["act"] == "relu" else x).T @ s["dy"][r: r + 32768].double()
    return {"dw": dw}


def _exact_table():
    """The 256 values of the e4m3 format: sign, four bits of exponent (bias 7), three of fraction."""
    b = torch.arange(256, device="cuda")
    e, m = (b >> 3) & 15, (b & 7).double()
    v = torch.where(e > 0, (1 + m / 8) * torch.exp2((e - 7).double()), m / 8 * 2.0 ** -6)
    return torch.where(b >= 128, -v, v)


def _exact_logits(s, case):
    R, scale, tokens, V = case["R"], case.get("scale", 1.0), s["tokens"], case["V"]
    rows = max(1, (1 << 27) // V)
    logp, ent = torch.zeros(R, dtype=torch.float64, device="cuda"), torch.zeros(R, dtype=torch.float64, device="cuda")
    counted = tokens >= 0

    def part(r):
        lp = torch.log_softmax(scale * s["logits"][r: r + rows].double(), 1)
        return lp, lp.exp(), tokens[r: r + rows].clamp(min=0)

    for r in range(0, R, rows):
        lp, p, t = part(r)
        logp[r: r + rows] = lp[torch.arange(len(t), device="cuda"), t]
        ent[r: r + rows] = -torch.xlogy(p, p).sum(1)
    logp, ent = logp.where(counted, logp.new_zeros(())), ent.where(counted, ent.new_zeros(()))
    out, h = {}, None
    if case["kind"] == "logp":
        out = {"logp": logp, "entropy": ent}
        g, h = s["dlogp"].double(), s["dentropy"].double()
        if not case["back"]:
            return out
    elif case["kind"] == "policy_grad":
        st, g, h = _exact_policy(s, case, logp, ent, counted)
        out = {"stats": st, "logp": logp, "entropy": ent}
    else:
        st, z, g = _exact_pairs(s, case, logp, counted)
        out = {"stats": st, "margin": z}
    d = torch.empty(R, V, dtype=torch.float64, device="cuda")
    for r in range(0, R, rows):
        lp, p, t = part(r)
        q = slice(r, r + rows)
        own_token = torch.arange(V, device="cuda") == t[:, None]
        v = g[q, None] * (own_token.double() - p)
        if h is not None:
            v = v - h[q, None] * (torch.xlogy(p, p) + p * ent[q, None])
        d[q] = (scale * v).where(counted[q, None], v.new_zeros(()))
    out["dlogits"] = d
    return out


def _exact_rows(s, R, seqs, counted):
    """The sequence of each row, and which rows count."""
    starts, at = s["offsets"][:-1], torch.arange(R, device="cuda")
    seq = torch.zeros(R, dtype=torch.long, device="cuda")
    for i in range(0, R, 1 << 16):
        seq[i: i + (1 << 16)] = (at[i: i + (1 << 16), None] >= starts).sum(1) - 1
    return seq, counted & (at < s["offsets"][-1])


def _exact_policy(s, case, logp, ent, counted):
    seq, counted = _exact_rows(s, case["R"], case["seqs"], counted)
    n = torch.bincount(seq[counted], minlength=case["seqs"]).double()
    if case["mean"] == "token":
        w = torch.full_like(logp, 1.0) / max(1.0, float(n.sum()))
    elif case["mean"] == "sequence":
        w = 1.0 / (n[seq] * max(1.0, float((n > 0).sum())))
    else:
        w = torch.full_like(logp, 1.0 / s["divisor"])
    w = w.where(counted, w.new_zeros(()))
    A, ratio = s["adv"].double(), (logp - s["old"].double()).exp()
    lo, hi = ratio * A, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * A
    gain = torch.minimum(lo, hi)
    flat = hi < lo
    if case["dual"]:
        flat = flat | ((A < 0) & (gain < case["dual"] * A))
        gain = gain.where(A >= 0, torch.maximum(gain, case["dual"] * A))
    g = (-lo).where(~flat, lo.new_zeros(()))
    kl = torch.zeros_like(logp)
    if s["ref"] is not None:
        z = logp - s["ref"].double()
        kl = {"k1": z, "k2": z.square() / 2, "k3": torch.expm1(-z) + z}[case["kl"]]
        g = g + KL_COEF * {"k1": torch.ones_like(z), "k2": z, "k3": -torch.expm1(-z)}[case["kl"]]
    total = lambda v: (w * v).where(counted, w.new_zeros(())).sum()  # noqa: E731
    t = [-total(gain), total(kl), total(ent), total(flat.double()), total(s["old"].double() - logp)]
    return (torch.stack([t[0] + KL_COEF * t[1] - ENTROPY_COEF * t[2], *t]), (w * g).where(counted, w.new_zeros(())), -ENTROPY_COEF * w)


def _exact_pairs(s, case, logp, counted):
    P = case["P"]
    seq, counted = _exact_rows(s, case["R"], 2 * P, counted)
    n = torch.bincount(seq[counted], minlength=2 * P).double()
    a = torch.bincount(seq[counted], weights=(logp - s["ref"].double())[counted], minlength=2 * P)
    per = 1.0 / n.clamp(min=1) if case["mean"] else torch.ones_like(n)
    reward = BETA * a * per
    there = (n[:P] * n[P:]) > 0
    z = reward[:P] - reward[P:] - MARGIN
    if case["loss"] == "sigmoid":
        ls = torch.nn.functional.logsigmoid
        loss, dz = -(1 - SMOOTHING) * ls(z) - SMOOTHING * ls(-z), torch.sigmoid(z) - (1 - SMOOTHING)
    elif case["loss"] == "hinge":
        loss, dz = (1 - z).relu(), torch.where(z < 1, -1.0, 0.0).double()
    else:
        h = (z / BETA) - 1 / (2 * BETA)
        loss, dz = h * h, 2 * h / BETA
    k = max(1, int(there.sum()))
    mean = lambda v: v[there].sum() / k  # noqa: E731
    st = torch.stack([mean(loss), mean((z > 0).double()), mean(reward[:P]), mean(reward[P:]), mean(z)])
    ds = (BETA / k * dz).where(there, dz.new_zeros(()))
    ds = torch.cat((ds, -ds)) * per
    return st, z.where(there, z.new_zeros(())), ds[seq].where(counted, ds.new_zeros(()))


def _exact_ckpt(s, case):
    dtype, K = s["x"].dtype, case["K"]
    table = _exact_table()[:127]  # the numbers from 0 to 448, in order
    y, kept, dx = (torch.empty(case["R"], K, dtype=torch.float64, device="cuda") for _ in range(3))
    step = max(1, (1 << 25) // K)
    for r in range(0, case["R"], step):
        x = s["x"][r: r + step].double()
        blocks = torch.nn.functional.pad(x, (0, -K % BLOCK)).view(x.shape[0], -1, BLOCK)
        top = blocks.abs().amax(2, keepdim=True)
        E = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448)).clamp(E_MIN, E_MAX)
        v = blocks / torch.exp2(E)
        hi = torch.searchsorted(table, v.abs()).clamp(max=126)  # the first number that is not smaller
        lo = (hi - 1).clamp(min=0)
        a, b = v.abs() - table[lo], table[hi] - v.abs()
        pick = torch.where((a < b) | ((a == b) & (lo % 2 == 0)), lo, hi)
        q = (torch.sign(v) * table[pick] * torch.exp2(E)).view(x.shape[0], -1)[:, :K]
        f, df = {"identity": (lambda u: u, torch.ones_like), "relu": (lambda u: u.relu(), lambda u: (u > 0).double()),
                 "silu": (torch.nn.functional.silu, lambda u: torch.sigmoid(u) * (1 + u * torch.sigmoid(-u))),
                 "gelu": (torch.nn.functional.gelu, lambda u: torch.special.ndtr(u) + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi))}[case["act"]]
        y[r: r + step], kept[r: r + step] = f(x), q.clamp(-torch.finfo(dtype).max, torch.finfo(dtype).max)
        dx[r: r + step] = s["dy"][r: r + step].double() * df(q)
    return {"y": y, "kept": kept, "dx": dx}


# ---------------------------------------------------------------------------------------------------------------------


def work(case):
    """What a pass cannot do without: inputs in, outputs out, each once; the arithmetic of a row's softmax as four operations a
    score forward and four more for its gradient."""
    kind, R = case["kind"], float(case["R"])
    es = 4.0 if case.get("dtype") == F32 else 2.0
    if kind == "logp":
        n, back = R * case["V"], case["back"]
        return {"bytes": n * es * (2 if back else 1) + R * (8 + 8 + (8 if back else 0)), "flops": n * (8 if back else 4)}
    if kind == "policy":
        return {"bytes": R * (4 * 5 + 1 + 8) + 8.0 * case["seqs"], "flops": R * 30}
    if kind == "policy_grad":
        n = R * case["V"]
        return {"bytes": n * es * 2 + R * (8 + 4 * 3 + 8) + 8.0 * case["seqs"], "flops": n * 8}
    if kind == "pairs":
        return {"bytes": R * (4 * 2 + 1 + 4) + 20.0 * case["P"], "flops": R * 4}
    if kind == "pairs_grad":
        n = R * case["V"]
        return {"bytes": n * es * 2 + R * (8 + 4) + 20.0 * case["P"], "flops": n * 8}
    if kind == "ckpt":
        n = R * case["K"]
        return {"bytes": n * (es * 5 + 1 + 1 / 32), "flops": n * 20}
    K, N = float(case["K"]), float(case["N"])
    return {"bytes": R * K * (1 + 1 / 32) + R * N * es + 4 * K * N, "flops": 2 * R * K * N}
