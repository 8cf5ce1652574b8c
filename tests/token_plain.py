"""The operators over token rows and the 8-bit checkpoints, written down from their formulas in 64 bits (torch, CPU or GPU)."""
import math

import torch

F64 = torch.float64


def counted_rows(rows, tokens=None, mask=None, offsets=None):
    """(counted, sequence of each row)."""
    dev = tokens.device if tokens is not None else offsets.device if offsets is not None else mask.device if mask is not None else "cpu"
    ok = torch.ones(rows, dtype=torch.bool, device=dev)
    if tokens is not None:
        ok &= tokens >= 0
    if mask is not None:
        ok &= mask != 0
    seq = torch.zeros(rows, dtype=torch.long, device=dev)
    if offsets is not None:
        r = torch.arange(rows, device=dev)
        seq = (r[:, None] >= offsets[None, :].long()).sum(1) - 1
        ok &= (seq >= 0) & (seq < offsets.numel() - 1)
    return ok, seq


def logp(logits, tokens, scale=1.0, mask=None):
    """logp, entropy, log of all probabilities; rows that do not count: zeros; a row of -inf: -inf and 0; tokens past the vocabulary: NaN."""
    R, V = logits.shape
    ok, _ = counted_rows(R, tokens, mask)
    x = logits.to(F64).clone()
    x[~ok] = 0.0
    none = (x == -math.inf).all(1)
    x[none] = 0.0
    lp = torch.log_softmax(scale * x, 1)
    p = lp.exp()
    H = -torch.xlogy(p, p).sum(1)
    l = lp.gather(1, tokens.long().clamp(0, V - 1)[:, None])[:, 0]
    l = torch.where(none, torch.full_like(l, -math.inf), l)
    l = torch.where(tokens.long() >= V, torch.full_like(l, math.nan), l)
    H = torch.where(none, torch.zeros_like(H), H)
    zero = torch.zeros_like(l)
    return torch.where(ok, l, zero), torch.where(ok, H, zero), lp, none


def dlogits(logits, tokens, dlogp, dentropy=None, scale=1.0, mask=None):
    R, V = logits.shape
    ok, _ = counted_rows(R, tokens, mask)
    _, H, lp, none = logp(logits, tokens, scale, mask)
    p = lp.exp()
    hot = torch.nn.functional.one_hot(tokens.long().clamp(0, V - 1), V).to(F64)
    g = dlogp.to(F64)[:, None] * (hot - p)
    if dentropy is not None:
        g -= dentropy.to(F64)[:, None] * (torch.xlogy(p, p) + p * H[:, None])
    g = torch.where((none | ~ok)[:, None], torch.zeros_like(g), scale * g)
    return torch.where((ok & ~none & (tokens.long() >= V))[:, None], torch.full_like(g, math.nan), g)


def policy(obj, l, old, adv, ref=None, H=None, tokens=None, mask=None, offsets=None):
    """stats, dlogp, dentropy of the clipped loss; obj: a dict of the objective's fields with kl and mean by name."""
    R = l.numel()
    ok, seq = counted_rows(R, tokens, mask, offsets)
    ok = ok.to(l.device)
    seq = seq.to(l.device)
    S = 1 if offsets is None else offsets.numel() - 1
    n = torch.bincount(seq[ok], minlength=max(S, 1)).to(F64)
    w = torch.zeros(R, dtype=F64, device=l.device)
    if obj["mean"] == "token":
        w[ok] = 1.0 / max(1, int(ok.sum()))
    elif obj["mean"] == "sequence":
        w[ok] = 1.0 / (n[seq[ok]] * max(1, int((n > 0).sum())))
    else:
        w[ok] = 1.0 / obj["divisor"]
    z = torch.zeros(R, dtype=F64, device=l.device)
    l = torch.where(ok, l.to(F64), z)
    A = torch.where(ok, adv.to(F64), z)
    d = torch.where(ok, l - old.to(F64), z) if old is not None else z
    r = d.clamp(-80, 80).exp()
    gain, cl = r * A, r.clamp(1 - obj["clip_low"], 1 + obj["clip_high"]) * A
    cut = cl < gain
    pg = -torch.minimum(gain, cl)
    if obj["dual_clip"]:
        over = (A < 0) & (pg > -obj["dual_clip"] * A)
        pg, cut = torch.where(over, -obj["dual_clip"] * A, pg), cut | over
    g = torch.where(cut, z, -gain)
    kl = z
    if obj["kl"] != "none":
        y = torch.where(ok, l - ref.to(F64), z)
        kl = {"k1": y, "k2": y * y / 2, "k3": torch.expm1(-y) + y}[obj["kl"]]
        g = g + obj["kl_coef"] * {"k1": torch.ones_like(y), "k2": y, "k3": -torch.expm1(-y)}[obj["kl"]]
    Hs = torch.where(ok, H.to(F64), z) if H is not None else z
    t = [(w * v).sum() for v in (pg, kl, Hs, cut.to(F64), -d)]
    k = obj["kl_coef"] if obj["kl"] != "none" else 0.0
    stats = torch.stack([t[0] + k * t[1] - obj["entropy_coef"] * t[2], *t])
    return stats, w * g, (-obj["entropy_coef"] * w if H is not None else None)


def preference(kind, beta, margin, smoothing, mean, l, offsets, ref=None, tokens=None, mask=None):
    R, P = l.numel(), (offsets.numel() - 1) // 2
    ok, seq = counted_rows(R, tokens, mask, offsets)
    a = torch.zeros(2 * P, dtype=F64, device=l.device)
    n = torch.zeros(2 * P, dtype=F64, device=l.device)
    for s in range(2 * P):
        at = ok & (seq == s)
        n[s] = at.sum()
        a[s] = (l.to(F64) - (ref.to(F64) if ref is not None else 0.0))[at].sum()
    if mean:
        a = a / n.clamp(min=1)
    there = (n[:P] > 0) & (n[P:] > 0)
    z = torch.where(there, beta * (a[:P] - a[P:]) - margin, torch.zeros(P, dtype=F64, device=l.device)).requires_grad_()
    ls = torch.nn.functional.logsigmoid
    loss = {"sigmoid": lambda: -(1 - smoothing) * ls(z) - smoothing * ls(-z), "hinge": lambda: (1 - z).clamp(min=0), "squared": lambda: ((z - 0.5) / beta) ** 2}[kind]()
    k = max(1, int(there.sum()))
    total = loss[there].sum() / k
    dz = torch.autograd.grad(total, z)[0] if there.any() else torch.zeros_like(z)
    z = z.detach()
    m = lambda v: v[there].sum() / k  # noqa: E731
    stats = torch.stack([total.detach(), m((z > 0).to(F64)), m(beta * a[:P]), m(beta * a[P:]), m(z)])
    da = torch.cat((beta * dz, -beta * dz))
    if mean:
        da = da / n.clamp(min=1)
    g = torch.zeros(R, dtype=F64, device=l.device)
    g[ok] = da[seq[ok]] if P else 0.0
    return stats, z, g


def e4m3_values(device="cpu"):
    """The numbers of the format from 0 to 448, ascending."""
    b = torch.arange(127, device=device)
    e, m = b >> 3, (b & 7).to(F64)
    return torch.where(e > 0, (1 + m / 8) * torch.exp2((e - 7).to(F64)), m / 8 * 2.0 ** -6)


def kept(x):
    """What an 8-bit checkpoint gives back for x (in 64 bits), and the scale exponents."""
    R, K = x.shape
    v = torch.nn.functional.pad(x.to(F64), (0, -K % 32)).reshape(R, -1, 32)
    fin = torch.isfinite(v)
    top = torch.where(fin, v.abs(), torch.zeros_like(v)).amax(2, keepdim=True)
    f, e = torch.frexp(top)
    E = torch.where(f > 0.875, e - 8, e - 9)
    E = torch.where(top > 0, E, torch.full_like(E, -117)).clamp(-117, 120)
    q = torch.where(fin, v, torch.zeros_like(v)) * torch.exp2(-E.to(F64))
    table = e4m3_values(x.device)
    hi = torch.searchsorted(table, q.abs().contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    a, b = q.abs() - table[lo], table[hi] - q.abs()
    pick = table[torch.where((a < b) | ((a == b) & (lo % 2 == 0)), lo, hi)]
    pick = torch.where(E == 120, pick.clamp(max=240), pick)
    out = torch.sign(q) * pick * torch.exp2(E.to(F64))
    out = torch.where(fin, out, torch.full_like(out, math.nan))
    return out.reshape(R, -1)[:, :K], E[:, :, 0]


def act(name, x):
    if name == "relu":
        return torch.where(x > 0, x, torch.where(x.isnan(), x, torch.zeros_like(x)))
    if name == "silu":
        return x * torch.sigmoid(x)
    if name == "gelu":
        return x * torch.special.ndtr(x)
    return x


def slope(name, x):
    if name == "relu":
        return torch.where(x.isnan(), x, (x > 0).to(F64))
    if name == "silu":
        s = torch.sigmoid(x)
        return s * (1 + x * (1 - s))
    if name == "gelu":
        return torch.special.ndtr(x) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    return torch.ones_like(x)
