"""Operators over token rows on the GPU against their formulas in 64 bits: log-probability and entropy, the gradient of the logits, the
clipped policy loss (from log-probabilities and from logits) and the preference loss.

Tolerances.  A probability p_j = 2^(c (x_j - m)) / s is off by the exponent's rounding (2^-23 of it), the exponential's 2^-22 and the sum's: a
thread adds at most V/32 + 8 terms (V/256 + 8 in rows that a whole block takes), each addition off by 2^-24 of the running sum.  With D the largest
|log p| that counts: rel = 2^-22 (2 + D) + 2^-24 (V/32 + 16).  log p itself is a difference of numbers of its own size: 2^-22 (|log p| + ln V + 1)
on top.  An output of a 16-bit type is rounded once: eps/2 of itself."""
import math

import pytest
import torch

from tests import token_plain as plain

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def tk():
    from paper_2104_06272_b200 import tokens

    return tokens


def rel_of(V, D=20.0):
    return 2.0 ** -22 * (2 + D) + 2.0 ** -24 * (V / 32 + 16)


def tol_logp(V, l):
    l = l.abs().nan_to_num(posinf=0.0, neginf=0.0)
    return rel_of(V) + 2.0 ** -22 * (l + math.log(V) + 1)


def half(dtype):
    return torch.finfo(dtype).eps / 2 if dtype != torch.float32 else 0.0


def tiny(dtype):
    """Half a step of the smallest numbers of the type."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


def near(got, want, tol):
    got, want = got.double(), want.double()
    same = (got == want) | (got.isnan() & want.isnan())
    tol = torch.as_tensor(tol, dtype=torch.float64, device=got.device).expand_as(want)
    bad = ~same & ~((got - want).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, the first at {bad.nonzero()[0].tolist()}: {got[bad][0].item()} for {want[bad][0].item()}, tolerance {tol[bad][0].item()}"


def make(R, V, dtype, seed=0, pad=0, shift=0, spread=2.5, ignored=0.0):
    """Logits in rows V + pad apart, `shift` elements into an allocation, NaN in the gaps; tokens int64."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((shift + R * (V + pad) + 8,), math.nan, dtype=dtype, device="cuda")
    x = flat[shift: shift + R * (V + pad)].view(R, V + pad)[:, :V]
    x.copy_(torch.randn(R, V, generator=g, device="cuda") * spread)
    tokens = torch.randint(0, V, (R,), generator=g, device="cuda")
    tokens[torch.rand(R, generator=g, device="cuda") < ignored] = -100
    return x, tokens, g


def check_rows(tk, x, tokens, scale=1.0, mask=None, g=None):
    R, V = x.shape
    o = tk.logp(x, tokens, scale=scale, mask=mask)
    l, H, lp, none = plain.logp(x, tokens, scale, mask)
    near(o.logp, l, tol_logp(V, l))
    # H = ln s - ln2 t/s: two numbers of about ln V
    near(o.entropy, H, rel_of(V) * (1 + math.log(V)) + 2.0 ** -22 * (math.log(V) + 1))
    lse = scale * o.norm[:, 0].double() + o.norm[:, 1].double()
    ok, _ = plain.counted_rows(R, tokens, mask)
    want = torch.logsumexp(scale * x.double(), 1)
    near(lse[ok & ~none], want[ok & ~none], 2.0 ** -22 * (want[ok & ~none].abs() + math.log(V) + 2) + rel_of(V))
    dl = torch.randn(R, generator=g, device="cuda")
    dh = torch.randn(R, generator=g, device="cuda")
    for ent in (False, True):
        got = tk.logp_backward(x, tokens, o.norm, dl, entropy=o.entropy if ent else None, dentropy=dh if ent else None, scale=scale, mask=mask)
        ref = plain.dlogits(x, tokens, dl, dh if ent else None, scale, mask)
        size = scale * (dl.abs() + (dh.abs() * (2 + math.log(V)) if ent else 0.0)).double()[:, None]
        near(got, ref, half(x.dtype) * ref.abs() + tiny(x.dtype) + rel_of(V) * size)
        # in place
        y = x.clone(memory_format=torch.preserve_format) if x.is_contiguous() else x
        if y is not x:
            tk.logp_backward(y, tokens, o.norm, dl, entropy=o.entropy if ent else None, dentropy=dh if ent else None, scale=scale, mask=mask, out=y)
            assert torch.equal(y.nan_to_num(), got.nan_to_num())
    return o


@pytest.mark.parametrize("V", [1, 2, 3, 4, 5, 8, 9, 31, 64, 128, 129, 1000, 2047, 2048, 2049, 5003, 32003])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_logp_and_its_gradient(tk, V, dtype):
    for R, pad, shift in ((1, 0, 0), (37, 0, 0), (13, 3, 1), (300, 8, 0)):
        x, tokens, g = make(R, V, DT[dtype], V + R, pad, shift, ignored=0.2 if R > 1 else 0.0)
        check_rows(tk, x, tokens, scale=0.7 if pad else 1.0, g=g)


@pytest.mark.parametrize("R,V", [(1, 200001), (3, 131072), (149, 70000), (2, 262144)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_rows(tk, R, V, dtype):
    x, tokens, g = make(R, V, DT[dtype], R, 0, 0, ignored=0.0)
    check_rows(tk, x, tokens, g=g)


@pytest.mark.parametrize("V", [4, 100, 1000, 5000, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_masks_of_the_vocabulary(tk, V, dtype):
    """-inf and the type's lowest value among the logits, rows of nothing else, one-token rows, large logits."""
    x, tokens, g = make(12, V, DT[dtype], V)
    low = torch.finfo(DT[dtype]).min
    x[0, torch.rand(V, generator=g, device="cuda") < 0.5] = -math.inf
    x[1, torch.rand(V, generator=g, device="cuda") < 0.5] = low
    x[2] = -math.inf
    x[3] = low
    x[4] = -math.inf
    x[4, V // 2] = 3.0
    x[5] = -math.inf
    x[5, tokens[5]] = 1.0
    x[6] *= 300.0  # far apart
    x[7] += 1000.0 if dtype != "f16" else 100.0  # a large common part
    x[8] = 0.0
    x[9, tokens[9]] = -math.inf  # the taken token has no probability
    x[10] = low
    x[10, 0] = -low
    l = plain.logp(x, tokens)[0].float()  # (row 10 of fp32: the lowest value less the highest is -6.8e38, which rounds to -inf)
    # (differences up to twice the type's largest: log p of -1e5 and below is compared in its own size)
    o = tk.logp(x, tokens)
    near(o.logp, l, tol_logp(V, l) + 2.0 ** -22 * l.abs().nan_to_num(posinf=0.0, neginf=0.0))
    assert o.logp[2].item() == -math.inf and o.entropy[2].item() == 0.0
    assert o.logp[9].item() == (-math.inf if V > 1 else o.logp[9].item())
    near(o.entropy, plain.logp(x, tokens)[1], rel_of(V) * (1 + math.log(V)) + 2.0 ** -22 * (math.log(V) + 1))
    dl, dh = torch.randn(12, generator=g, device="cuda"), torch.randn(12, generator=g, device="cuda")
    got = tk.logp_backward(x, tokens, o.norm, dl, entropy=o.entropy, dentropy=dh)
    ref = plain.dlogits(x, tokens, dl, dh)
    near(got, ref, half(x.dtype) * ref.abs() + tiny(x.dtype) + rel_of(V) * (dl.abs() + dh.abs() * (2 + math.log(V))).double()[:, None])
    assert (got[2] == 0).all()


@pytest.mark.parametrize("V", [4, 1000, 9000])
def test_rows_that_do_not_count_may_hold_anything(tk, V):
    x, tokens, g = make(9, V, torch.float32, 5)
    mask = torch.ones(9, dtype=torch.bool, device="cuda")
    mask[2] = False
    tokens[4] = -1
    clean = tk.logp(x, tokens, mask=mask)
    d = torch.randn(9, generator=g, device="cuda")
    want = tk.logp_backward(x, tokens, clean.norm, d, entropy=clean.entropy, dentropy=d, mask=mask)
    for bad in (math.nan, math.inf, -math.inf):
        x[2], x[4] = bad, bad
        o = tk.logp(x, tokens.int(), mask=mask.to(torch.uint8))
        assert all(torch.equal(a, b) for a, b in zip(o, clean)) and o.logp[2] == 0 and o.entropy[4] == 0
        d[2], d[4] = bad, bad
        got = tk.logp_backward(x, tokens, o.norm, d, entropy=o.entropy, dentropy=d, mask=mask)
        assert torch.equal(got, want) and (got[2] == 0).all() and (got[4] == 0).all()


@pytest.mark.parametrize("V", [4, 700, 3000])
def test_nan_and_tokens_past_the_vocabulary_are_seen(tk, V):
    x, tokens, g = make(6, V, torch.float32, 3)
    x[1, V - 1] = math.nan
    x[2, 0] = math.inf
    tokens[3] = V
    tokens[4] = (1 << 40) + 1
    o = tk.logp(x, tokens)
    assert o.logp[1:5].isnan().all() and o.logp[[0, 5]].isfinite().all() and o.entropy[[0, 3, 4, 5]].isfinite().all()
    got = tk.logp_backward(x, tokens, o.norm, torch.ones(6, device="cuda"))
    assert got[1:5].isnan().any(1).all() and got[[0, 5]].isfinite().all()


def objective(tk, **kw):
    f = dict(clip_low=0.2, clip_high=0.28, dual_clip=0.0, kl="k3", kl_coef=0.05, entropy_coef=0.01, mean="token", divisor=100.0)
    f.update(kw)
    return f, tk.policy_objective(**f)


def policy_inputs(R, S, g, behind=0):
    l = -torch.rand(R, generator=g, device="cuda") * 5
    old = l + 0.2 * torch.randn(R, generator=g, device="cuda")
    ref = l + 0.3 * torch.randn(R, generator=g, device="cuda")
    adv = torch.randn(R, generator=g, device="cuda")
    H = torch.rand(R, generator=g, device="cuda")
    cuts = torch.randint(0, R - behind + 1, (S - 1,), generator=g, device="cuda").sort().values
    offsets = torch.cat((torch.zeros(1, dtype=torch.int64, device="cuda"), cuts, torch.tensor([R - behind], device="cuda")))
    mask = torch.rand(R, generator=g, device="cuda") > 0.3
    return l, old, adv, ref, H, offsets, mask


def off_the_edge(obj, l, old):
    """No ratio within rounding of a clip (there either side of the decision is right)."""
    r = (l.double() - old.double()).exp()
    for e in (1 - obj["clip_low"], 1 + obj["clip_high"], obj["dual_clip"] or 9.0):
        old = torch.where((r / e - 1).abs() < 1e-4, old + 1e-2, old)
    return old


def check_policy(got, want, R, amax):
    """Terms are formed in fp32 from r = exp(d), |d| <= 2: off by less than 2^-20 of r A; sums of R of them in 64 bits, rounded once."""
    stats, dlogp, dent = want
    near(got.dlogp, dlogp, 2.0 ** -20 * dlogp.abs() + 2.0 ** -20 * dlogp.abs().max())
    near(got.stats, stats, 2.0 ** -19 * (1 + amax))
    if dent is not None:
        near(got.dentropy, dent, 2.0 ** -22 * dent.abs())


@pytest.mark.parametrize("mean", ["token", "sequence", "fixed"])
@pytest.mark.parametrize("kl,dual", [("none", 0.0), ("k1", 3.0), ("k2", 0.0), ("k3", 1.5)])
@pytest.mark.parametrize("R,S", [(1, 1), (33, 7), (1000, 40), (8192, 9), (8193, 300), (20000, 5000), (70001, 1)])
def test_policy_loss(tk, R, S, kl, dual, mean):
    g = torch.Generator(device="cuda").manual_seed(R + S)
    l, old, adv, ref, H, offsets, mask = policy_inputs(R, S, g, R // 10)
    f, obj = objective(tk, kl=kl, dual_clip=dual, mean=mean)
    old = off_the_edge(f, l, old)
    if R <= 33:
        mask[:] = True
    l[~mask], adv[~mask], H[~mask] = math.nan, math.inf, math.nan
    got = tk.policy_loss(obj, l, old, adv, ref_logp=ref if kl != "none" else None, entropy=H, mask=mask, offsets=offsets if R % 2 else offsets.int())
    want = plain.policy(f, l, old, adv, ref, H, None, mask, offsets)
    check_policy(got, want, R, float(adv[mask].abs().max()) * 10)
    again = tk.policy_loss(obj, l, old, adv, ref_logp=ref if kl != "none" else None, entropy=H, mask=mask, offsets=offsets)
    assert torch.equal(again.stats, got.stats) and torch.equal(again.dlogp, got.dlogp)


def test_policy_loss_corners(tk):
    f, obj = objective(tk, entropy_coef=0.0)
    R = 12
    l = torch.tensor([-1.0] * R, device="cuda")
    old, adv, ref = l.clone(), torch.ones(R, device="cuda"), l.clone()
    old[0], adv[0] = l[0] + 200.0, 0.0      # ratio to nothing
    old[1], adv[1] = l[1] - 200.0, 1.0      # ratio beyond any number: clipped
    old[2], adv[2] = l[2] - 200.0, 0.0      # the same without advantage
    l[3] = -math.inf                        # the policy has given the token up
    ref[3] = -math.inf
    ref[4] = l[4] + 1e-4                    # a small difference: exp(-z) - 1 + z is about z^2 / 2
    adv[5] = 0.0
    got = tk.policy_loss(obj, l, old, adv, ref_logp=ref, mask=torch.arange(R, device="cuda") != 3)
    want = plain.policy(f, l, old, adv, ref, None, None, torch.arange(R, device="cuda") != 3)
    check_policy(got, want, R, 2.0)
    one = tk.policy_loss(obj, l[4:5].clone(), old[4:5].clone(), torch.zeros(1, device="cuda"), ref_logp=ref[4:5].clone())
    z = (l[4].double() - ref[4].double()).item()
    assert abs(one.stats[2].item() - (math.expm1(-z) + z)) <= 2.0 ** -20 * z * z
    # without an old policy the ratio is one and its gradient is there
    on = tk.policy_loss(objective(tk, kl="none")[1], l, None, adv)
    near(on.dlogp, -adv.double() / R, 1e-8)
    # nothing counts, or there is nothing
    none = tk.policy_loss(obj, l, old, adv, ref_logp=ref, mask=torch.zeros(R, dtype=torch.bool, device="cuda"))
    assert (none.stats == 0).all() and (none.dlogp == 0).all()
    e = torch.empty(0, device="cuda")
    assert (tk.policy_loss(obj, e, e, e, ref_logp=e).stats == 0).all()
    for mean in ("token", "sequence"):
        z0 = tk.policy_loss(objective(tk, mean=mean)[1], l, old, adv, ref_logp=ref, offsets=torch.zeros(1, dtype=torch.int64, device="cuda"))
        assert (z0.stats == 0).all() and (z0.dlogp == 0).all()


@pytest.mark.parametrize("mean,kl", [("token", "k3"), ("sequence", "none"), ("fixed", "k2")])
@pytest.mark.parametrize("R,V,pad", [(1, 1, 0), (40, 4, 0), (257, 5, 2), (30, 100, 0), (100, 1500, 1), (37, 5000, 0), (70, 32003, 0), (5, 131072, 0), (150, 50000, 8)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_policy_grad_is_the_three_calls(tk, R, V, pad, dtype, mean, kl):
    x, tokens, g = make(R, V, DT[dtype], R + V, pad, 0, ignored=0.25 if R > 1 else 0.0)
    S = min(R, 6)
    _, _, adv, _, _, offsets, _ = policy_inputs(R, S, g, R // 8)
    f, obj = objective(tk, mean=mean, kl=kl)
    l = plain.logp(x, tokens, 0.9)[0]
    old = off_the_edge(f, l, (l + 0.2 * torch.randn(R, generator=g, device="cuda")).float())
    ref = (l + 0.2 * torch.randn(R, generator=g, device="cuda")).float()
    got = tk.policy_grad(obj, x, tokens, old, adv, ref_logp=ref if kl != "none" else None, offsets=offsets, scale=0.9)
    lp, H, _, _ = plain.logp(x, tokens, 0.9)
    stats, dl, dh = plain.policy(f, lp, old, adv, ref, H, tokens, None, offsets)
    near(got.logp, lp, tol_logp(V, lp))
    amax = float(adv.abs().max())
    # (log p is off by its tolerance, and so, relative, is the ratio)
    near(got.stats, stats, (2.0 ** -19 + 4 * float(tol_logp(V, lp).max())) * (2 + amax + math.log(V)))
    want = plain.dlogits(x, tokens, dl, dh, 0.9)
    size = (dl.abs() + dh.abs() * (2 + math.log(V)))[:, None]
    slack = (2.0 ** -20 + 3 * tol_logp(V, lp) + rel_of(V))[:, None] * (size + dl.abs().max())
    near(got.dlogits, want, half(x.dtype) * want.abs() + tiny(x.dtype) + slack)
    # the three calls give the same numbers
    o = tk.logp(x, tokens, scale=0.9)
    p = tk.policy_loss(obj, o.logp, old, adv, ref_logp=ref if kl != "none" else None, entropy=o.entropy, tokens=tokens, offsets=offsets)
    d = tk.logp_backward(x, tokens, o.norm, p.dlogp, entropy=o.entropy, dentropy=p.dentropy, scale=0.9)
    near(got.dlogits, d, 2 * half(x.dtype) * d.abs().double() + tiny(x.dtype) + slack)
    if x.is_contiguous():
        y = x.clone()
        z = tk.policy_grad(obj, y, tokens, old, adv, ref_logp=ref if kl != "none" else None, offsets=offsets, scale=0.9, out=y)
        assert torch.equal(y, got.dlogits) and torch.equal(z.stats, got.stats)


@pytest.mark.parametrize("scale", [1e-3, 40.0, 1e4, 2.0 ** 40])
@pytest.mark.parametrize("V", [3, 200, 6000])
def test_temperatures(tk, V, scale):
    """Logits whose scaled differences are of ordinary size, shifted by thousands of them."""
    x, tokens, g = make(8, V, torch.float32, V)
    x /= scale
    x[4:] += 16.0 / scale
    l, H, _, _ = plain.logp(x, tokens, scale)
    o = tk.logp(x, tokens, scale=scale)
    near(o.logp, l, tol_logp(V, l) + 2.0 ** -22 * 40)  # (the exponent's products are of size 40)
    near(o.entropy, H, rel_of(V) * (1 + math.log(V)) + 2.0 ** -22 * (math.log(V) + 1))


def test_no_rows(tk):
    x = torch.empty(0, 50, device="cuda")
    t, e = torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    o = tk.logp(x, t)
    assert o.logp.numel() == 0 and tk.logp_backward(x, t, o.norm, e).shape == (0, 50)
    f, obj = objective(tk)
    p = tk.policy_grad(obj, x, t, e, e, ref_logp=e)
    assert (p.stats == 0).all() and p.dlogits.shape == (0, 50)
    assert tk.logp(logits=torch.zeros(2, 4, device="cuda"), tokens=torch.zeros(2, dtype=torch.int64, device="cuda")).logp.shape == (2,)


def test_a_first_call_may_be_a_captured_one(tk, tmp_path):
    """In a process of its own, where no kernel of these has run."""
    import subprocess
    import sys

    code = """
import torch
from paper_2104_06272_b200 import tokens as tk
x = torch.randn(40, 30000, device="cuda", dtype=torch.bfloat16)
t = torch.randint(0, 30000, (40,), device="cuda")
a = torch.randn(40, device="cuda")
h = torch.randn(300, 200, device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    o = tk.policy_grad(tk.policy_objective(), x, t, None, a)
    y, ck = tk.ckpt_forward(h)
    w = tk.ckpt_weight_grad(ck, h, "relu")
g.replay()
torch.cuda.synchronize()
p = tk.policy_grad(tk.policy_objective(), x, t, None, a)
assert torch.equal(o.dlogits, p.dlogits) and torch.equal(w, tk.ckpt_weight_grad(ck, h, "relu"))
"""
    import os

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


def test_columns_behind_the_vocabulary_stay(tk):
    x, tokens, g = make(20, 5001, torch.bfloat16, 1)
    out = torch.full((20, 5016), 7.0, dtype=torch.bfloat16, device="cuda")
    o = tk.logp(x, tokens)
    tk.logp_backward(x, tokens, o.norm, torch.ones(20, device="cuda"), out=out[:, :5001])
    assert (out[:, 5001:] == 7).all() and (out[:, :5001] != 7).all()


def test_gradients_are_differences(tk):
    """Loss along a direction: (L(x + e v) - L(x - e v)) / 2e with e = 1/64.  The third derivative of these losses along a unit-sized v is
    below 10 of the first's scale: e^2/6 of that, and fp32 statistics' 2^-24 / e."""
    x, tokens, g = make(24, 600, torch.float32, 11, ignored=0.2)
    f, obj = objective(tk, mean="sequence")
    offsets = torch.tensor([0, 5, 5, 17, 22], device="cuda")
    l = tk.logp(x, tokens).logp
    old, ref = l + 0.05 * torch.randn(24, generator=g, device="cuda"), l + 0.2 * torch.randn(24, generator=g, device="cuda")
    adv = torch.randn(24, generator=g, device="cuda")
    v = torch.randn(24, 600, generator=g, device="cuda") * 0.2
    e = 1.0 / 64

    def loss(y):
        return tk.policy_grad(obj, y, tokens, old, adv, ref_logp=ref, offsets=offsets)

    got = (loss(x).dlogits.double() * v.double()).sum().item()
    diff = (loss(x + e * v).stats[0].double() - loss(x - e * v).stats[0].double()).item() / (2 * e)
    assert abs(got - diff) <= e * e / 6 * 10 + 2.0 ** -22 / e
    po = tk.preference_objective("sigmoid", beta=0.3, smoothing=0.1)

    def pref(y):
        o = tk.logp(y, tokens)
        return o, tk.preference_loss(po, o.logp, offsets, ref_logp=ref, tokens=tokens)

    o, p = pref(x)
    d = tk.logp_backward(x, tokens, o.norm, p.dlogp)
    got = (d.double() * v.double()).sum().item()
    diff = (pref(x + e * v)[1].stats[0].double() - pref(x - e * v)[1].stats[0].double()).item() / (2 * e)
    assert abs(got - diff) <= e * e / 6 * 10 + 2.0 ** -22 / e


@pytest.mark.parametrize("kind", ["sigmoid", "hinge", "squared"])
@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("R,P", [(4, 1), (100, 20), (3000, 3), (9000, 1500), (50000, 2)])
def test_preference_loss(tk, R, P, mean, kind):
    g = torch.Generator(device="cuda").manual_seed(R * P)
    l, _, _, ref, _, offsets, mask = policy_inputs(R, 2 * P, g, R // 9)
    l[~mask] = math.nan
    if R == 4:
        offsets, mask = torch.tensor([0, 2, 4], device="cuda"), torch.ones(4, dtype=torch.bool, device="cuda")
        l = l.nan_to_num(-1.0)
    obj = tk.preference_objective(kind, beta=0.2, margin=0.1, smoothing=0.15, mean=mean)
    for r in (ref, None):
        if r is None and not mean:
            continue  # (sums without a reference: hundreds of thousands, where hinge and sigmoid are flat)
        got = tk.preference_loss(obj, l, offsets, ref_logp=r, mask=mask)
        # (fields of the objective are fp32)
        beta, margin, smoothing = float(obj.beta), float(obj.margin), float(obj.smoothing)
        st, z, d = plain.preference(kind, beta, margin, smoothing, mean, l.nan_to_num(0.0), offsets, r, None, mask)
        # everything is in 64 bits and rounded once
        near(got.stats, st, 2.0 ** -23 * st.abs() + 1e-12)
        near(got.margin, z, 2.0 ** -23 * z.abs() + 1e-12)
        near(got.dlogp, d, 2.0 ** -23 * d.abs() + 1e-12)


def test_preference_loss_corners(tk):
    obj = tk.preference_objective("sigmoid", beta=1.0)
    l = torch.tensor([-1.0, -2.0, -3.0, -4.0], device="cuda")
    # an empty answer, or one without a counted row: the pair carries no loss
    for offsets, mask in (([0, 2, 2], None), ([0, 2, 4], [True, True, False, False])):
        o = tk.preference_loss(obj, l, torch.tensor(offsets, device="cuda"), mask=None if mask is None else torch.tensor(mask, device="cuda"))
        assert (o.stats == 0).all() and (o.dlogp == 0).all() and (o.margin == 0).all()
    # differences beyond any exponential
    far = torch.tensor([0.0, -2000.0], device="cuda")
    o = tk.preference_loss(obj, far, torch.tensor([0, 1, 2], device="cuda"))
    assert o.stats[0].item() == 0.0 and o.margin[0].item() == 2000.0 and (o.dlogp == 0).all()
    o = tk.preference_loss(obj, far.flip(0), torch.tensor([0, 1, 2], device="cuda"))
    assert o.stats[0].item() == 2000.0 and o.dlogp.tolist() == [-1.0, 1.0]
    e = torch.empty(0, device="cuda")
    o = tk.preference_loss(obj, e, torch.zeros(1, dtype=torch.int64, device="cuda"))
    assert (o.stats == 0).all() and o.margin.numel() == 0
    # sums of many terms that nearly cancel
    n = 60000
    a = torch.full((2 * n,), -7.3, device="cuda")
    a[0] = -7.0
    o = tk.preference_loss(obj, a, torch.tensor([0, n, 2 * n], device="cuda"))
    want = float(torch.tensor(-7.0).double() - torch.tensor(-7.3).double())
    assert abs(o.margin[0].item() - want) < 1e-6


@pytest.mark.parametrize("V", [4, 5000, 60000])
def test_side_streams_and_captured_graphs(tk, V):
    x, tokens, g = make(65, V, torch.bfloat16, 2, ignored=0.2)
    f, obj = objective(tk, mean="sequence")
    l = tk.logp(x, tokens).logp
    old, adv, ref = l + 0.01, torch.randn(65, generator=g, device="cuda"), l - 0.1
    offsets = torch.tensor([0, 30, 30, 65], device="cuda")
    call = lambda: tk.policy_grad(obj, x, tokens, old, adv, ref_logp=ref, offsets=offsets)  # noqa: E731
    want = call()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = call()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    po = tk.preference_objective("hinge")
    poff = torch.tensor([0, 30, 65], device="cuda")
    eager = tk.preference_loss(po, l, poff, tokens=tokens)
    with torch.cuda.graph(graph):
        out = call()
        small = tk.policy_loss(obj, l, old, adv, ref_logp=ref, tokens=tokens, offsets=offsets)
        pref = tk.preference_loss(po, l, poff, tokens=tokens)
    for seed in (3, 4):
        y = make(65, V, torch.bfloat16, seed)[0]
        x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        fresh = call()
        assert all(torch.equal(a, b) for a, b in zip(out, fresh))
        assert all(torch.equal(a, b) for a, b in zip(pref, eager)) and small.stats.isfinite().all()


def test_offsets_of_any_kind_stay_within_bounds(tk):
    """Offsets are data: wrong ones give wrong numbers and nothing else."""
    R = 300
    g = torch.Generator(device="cuda").manual_seed(1)
    l, old, adv, ref, H, _, mask = policy_inputs(R, 3, g)
    x, tokens, _ = make(R, 50, torch.float32)
    for off in ([0, 500, 100], [-5, 20, 1 << 40], [200, 100, 0], [300, 300, 300], [5, 5, 5]):
        o = torch.tensor(off, device="cuda")
        for mean in ("token", "sequence", "fixed"):
            obj = objective(tk, mean=mean)[1]
            tk.policy_loss(obj, l, old, adv, ref_logp=ref, entropy=H, offsets=o)
            tk.policy_grad(obj, x, tokens, old, adv, ref_logp=ref, offsets=o)
        p = tk.preference_loss(tk.preference_objective(), l, o)
        assert p.dlogp.isfinite().all()
    torch.cuda.synchronize()


def test_rows_past_32_bits(tk):
    """A matrix of more than 2^32 elements: the last rows are the ones that a short offset would miss."""
    R, V = 35000, 131072
    x = torch.zeros(R, V, dtype=torch.bfloat16, device="cuda")
    tokens = torch.zeros(R, dtype=torch.int64, device="cuda")
    x[-1] = torch.randn(V, device="cuda")
    tokens[-1] = 77
    o = tk.logp(x, tokens)
    l, H, _, _ = plain.logp(x[-1:], tokens[-1:])
    near(o.logp[-1:], l, tol_logp(V, l))
    near(o.logp[:1], torch.tensor([-math.log(V)], device="cuda"), tol_logp(V, torch.tensor([12.0], device="cuda")))
    d = torch.ones(R, device="cuda")
    tk.logp_backward(x, tokens, o.norm, d, out=x)
    want = plain.dlogits(torch.zeros(1, V, device="cuda"), tokens[:1], d[:1])
    near(x[-2:-1], want, 2.0 ** -8 * want.abs() + 1e-9)


def test_refusals_of_tensors(tk):
    """Types, shapes, strides and devices that do not fit; nothing is enqueued and the next call is sound."""
    x, tokens, _ = make(6, 10, torch.float32)
    v, w = torch.zeros(6, device="cuda"), torch.zeros(12, device="cuda")[::2]
    obj, po, off = tk.policy_objective(), tk.preference_objective(), torch.tensor([0, 3, 6], device="cuda")
    kl = tk.policy_objective(kl="k3", kl_coef=0.1)
    want = tk.logp(x, tokens)
    norm = want.norm
    calls = [
        lambda: tk.logp(None, tokens), lambda: tk.logp(x.double(), tokens), lambda: tk.logp(x.t(), tokens), lambda: tk.logp(x[:, :0], tokens), lambda: tk.logp(x[0], tokens),
        lambda: tk.logp(x, None), lambda: tk.logp(x, tokens[:5]), lambda: tk.logp(x, tokens.cpu()), lambda: tk.logp(x, tokens.float()), lambda: tk.logp(x, tokens.view(2, 3)),
        lambda: tk.logp(x, tokens, mask=v), lambda: tk.logp(x, tokens, 0.0), lambda: tk.logp(x, tokens, 1e300), lambda: tk.logp(x.expand(6, 10)[:1].expand(6, 10), tokens),
        lambda: tk.logp_backward(x, tokens, norm, None), lambda: tk.logp_backward(x, tokens, norm[:5], v), lambda: tk.logp_backward(x, tokens, norm, w),
        lambda: tk.logp_backward(x, tokens, norm, v, None, v), lambda: tk.logp_backward(x, tokens, norm, v, out=x.half()), lambda: tk.logp_backward(x, tokens, norm, v, out=x[:5]),
        lambda: tk.logp_backward(x, tokens, torch.zeros(6, 4, device="cuda")[:, :2], v), lambda: tk.policy_loss(obj, x, v, v), lambda: tk.policy_loss(obj, v, v, None),
        lambda: tk.policy_loss(kl, v, v, v), lambda: tk.policy_loss(po, v, v, v), lambda: tk.policy_loss(obj, v, v, v, offsets=off[:0]),
        lambda: tk.policy_loss(obj, v, v, v, offsets=off.view(1, 3)), lambda: tk.policy_grad(obj, x, None, v, v), lambda: tk.policy_grad(kl, x, tokens, v, v),
        lambda: tk.policy_grad(obj, x, tokens, v, v.half()), lambda: tk.preference_loss(obj, v, off), lambda: tk.preference_loss(po, v, None),
        lambda: tk.preference_loss(po, v, off[:2]), lambda: tk.preference_loss(po, v.half(), off)]
    for i, call in enumerate(calls):
        with pytest.raises(tk.AnakinError) as e:
            call()
            print(f"call {i} was taken")
        assert e.value.code == -1, i
    for call in (lambda: tk.logp(x, tokens, "1"), lambda: tk.policy_loss(None, v, v, v)):
        with pytest.raises(TypeError):
            call()
    again = tk.logp(x, tokens)
    assert all(torch.equal(a, b) for a, b in zip(want, again))


def test_two_threads_on_streams_of_their_own(tk):
    """Calls from several host threads at once share nothing."""
    import threading

    x, tokens, g = make(700, 3000, torch.bfloat16, 5, ignored=0.2)
    obj = tk.policy_objective(mean="sequence")
    adv = torch.randn(700, generator=g, device="cuda")
    offsets = torch.tensor([0, 400, 700], device="cuda")
    want = tk.policy_grad(obj, x, tokens, None, adv, offsets=offsets)
    torch.cuda.synchronize()
    bad = []

    def work():
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(20):
                got = tk.policy_grad(obj, x, tokens, None, adv, offsets=offsets)
                s.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(want, got)):
                    bad.append(1)

    threads = [threading.Thread(target=work) for _ in range(3)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not bad


@pytest.mark.parametrize("scale", [1.0, 0.7, 1.3])
@pytest.mark.parametrize("R,V,dtype", [(4000, 9823, torch.float16), (4000, 300, torch.float32), (1500, 40000, torch.bfloat16)])
def test_logp_has_no_bias(tk, R, V, dtype, scale):
    """Sums over sequences of thousands of tokens keep what errors have in common.  Roundings are off by nothing on the average; the exponential's
    error is 2^-22 at most and may be alike in all rows: a bound for the mean, with five deviations of roundings of |l| < 32 (2^-20 / sqrt(3 R))."""
    x, tokens, _ = make(R, V, dtype, 11)
    s32 = torch.tensor(scale, dtype=torch.float32).double().item()
    l = plain.logp(x, tokens, s32)[0]
    err = (tk.logp(x, tokens, scale).logp.double() - l).mean().item()
    assert abs(err) < 2.0 ** -22 + 5 * 2.0 ** -20 / (3 * R) ** 0.5, err


def test_more_than_2_to_the_30_sequences(tk):
    """Nearly all of them empty: places in the offsets whose sum passes 2^31."""
    S, R = (1 << 30) + 5, 9000
    offsets = torch.zeros(S + 1, dtype=torch.int32, device="cuda")
    offsets[S - 1], offsets[S] = 4010, R
    g = torch.Generator(device="cuda").manual_seed(1)
    l, old, adv, ref, H, _, mask = policy_inputs(R, 2, g)
    f, obj = objective(tk, mean="sequence")
    old = off_the_edge(f, l, old)
    near_offsets = torch.tensor([0, 4010, R], device="cuda")
    got = tk.policy_loss(obj, l, old, adv, ref_logp=ref, entropy=H, mask=mask, offsets=offsets)
    check_policy(got, plain.policy(f, l, old, adv, ref, H, None, mask, near_offsets), R, float(adv[mask].abs().max()) * 10)
    x, tokens, _ = make(R, 5, torch.float32, 3)
    a, b = (tk.policy_grad(obj, x, tokens, old, adv, ref_logp=ref, mask=mask, offsets=o) for o in (offsets, near_offsets))
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_the_longest_vocabulary(tk):
    """2^31 - 1 logits in a row: a column's number plus a block's threads would pass 32 bits."""
    V = (1 << 31) - 1
    x = torch.zeros(1 + V + 8, dtype=torch.bfloat16, device="cuda")[1: 1 + V].view(1, V)
    tokens = torch.tensor([V - 1], device="cuda")
    o = tk.logp(x, tokens)
    # (the sums are counts, exact in fp32 up to 2^24 in every thread)
    assert abs(o.logp[0].item() + math.log(V)) < 1e-5 and abs(o.entropy[0].item() - math.log(V)) < 1e-5
    flat = torch.full((V + 17,), 7.0, dtype=torch.bfloat16, device="cuda")
    got = flat[3: 3 + V].view(1, V)
    tk.logp_backward(x, tokens, o.norm, torch.ones(1, device="cuda"), out=got)
    assert got[0, -1] == 1.0 and abs(got[0, 0].item() * V + 1.0) < 2.0 ** -8 and (got[0, :-1] == got[0, 0]).all()
    assert (flat[:3] == 7).all() and (flat[3 + V:] == 7).all()


def check_fused(tk, x, tokens, scale, g):
    """The clipped loss without an old policy (the ratio is one): its gradient is that of given gradients of log p and entropy."""
    R, V = x.shape
    adv = torch.randn(R, generator=g, device="cuda")
    got = tk.policy_grad(tk.policy_objective(entropy_coef=0.01, mean="fixed", divisor=float(R)), x, tokens, None, adv, scale=scale)
    l, H, _, _ = plain.logp(x, tokens, scale)
    near(got.logp, l, tol_logp(V, l))
    near(got.entropy, H, rel_of(V) * (1 + math.log(V)) + 2.0 ** -22 * (math.log(V) + 1))
    dl, dh = -adv.double() / R, torch.full((R,), -0.01 / R, dtype=torch.float64, device="cuda")
    want = plain.dlogits(x, tokens, dl, dh, scale)
    size = scale * (dl.abs() + dh.abs() * (2 + math.log(V)))[:, None]
    near(got.dlogits, want, half(x.dtype) * want.abs() + tiny(x.dtype) + (2.0 ** -20 + rel_of(V)) * size)
    assert (got.logp <= 0).all() and (got.entropy >= 0).all()
    return got


@pytest.mark.parametrize("far", [-1e4, -1e9, -1e10, -1e12, -1e15, -1e20, -1e26, 1e6, 2907270.0, 1e10])  # (2907270 log2(e) is about 2^22)
@pytest.mark.parametrize("R", [14, 161])
@pytest.mark.parametrize("V", [4, 100, 200, 1000, 9000, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_finite_masks_and_common_parts(tk, V, dtype, R, far):
    """Numbers as masks are added with, whole chunks of a row, and rows of nothing else: the largest logit times c has a rounding error of
    any size, which no exponential may see."""
    x, tokens, g = make(R, V, DT[dtype], V)
    x[0::7, : V // 2] += far
    x[1::7, V // 3:] += far
    x[2::7, torch.rand(V, generator=g, device="cuda") < 0.5] += far
    x[3::7] = far
    x[4::7] += far
    x[5::7, :-1] = far
    check_rows(tk, x, tokens, g=g)
    check_fused(tk, x, tokens, 1.0, g)


@pytest.mark.parametrize("scale", [0.7, 1e4, 1e6, 3e7, 1e8, 2.0 ** 40])
@pytest.mark.parametrize("V", [4, 100, 200, 1000, 9000, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ordinary_logits_at_any_scale(tk, V, dtype, scale):
    """Not divided by it: the largest logit times c is as large as the scale is.  Half of the rows took their likeliest token; some
    have a large part in common."""
    x, tokens, g = make(150, V, DT[dtype], V + 1)
    x[::3] -= 1e9
    tokens[::2] = x[::2].float().argmax(1)
    check_rows(tk, x, tokens, scale, g=g)
    check_fused(tk, x, tokens, scale, g)


@pytest.mark.parametrize("R", [1, 200, 700])
@pytest.mark.parametrize("V", [5, 100, 129, 500, 2000, 9000, 40000, 131072])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_no_probability_above_one(tk, V, dtype, R):
    """Rows whose token has nearly all the probability (exp(3.1) V is about the sum of the others): log p is at most 0 and the entropy at least 0."""
    x, tokens, g = make(R, V, DT[dtype], V + R)
    x[torch.arange(R, device="cuda"), tokens] = (math.log(V) + 3.1 + torch.linspace(2.0, 25.0, R, device="cuda")).to(x.dtype)
    l, H, _, _ = plain.logp(x, tokens)
    for o in (tk.logp(x, tokens), tk.policy_grad(tk.policy_objective(), x, tokens, None, torch.ones(R, device="cuda"))):
        near(o.logp, l, tol_logp(V, l))
        near(o.entropy, H, rel_of(V) * (1 + math.log(V)) + 2.0 ** -22 * (math.log(V) + 1))
        assert (o.logp <= 0).all() and (o.entropy >= 0).all()


@pytest.mark.parametrize("scale", [1.0, 1e9, 2.0 ** 40])
@pytest.mark.parametrize("V", [4, 100, 200, 1000, 9000, 40000])
def test_gradients_of_entropies_at_any_scale(tk, V, scale):
    """Scaled logits of ordinary size beside tokens without probability: -inf, the lowest value, and what lies between."""
    x, tokens, g = make(161, V, torch.float32, V + 2)
    x /= scale
    for i, low in enumerate((-math.inf, torch.finfo(torch.float32).min, -1e15, -1e22)):
        x[i::5, torch.rand(V, generator=g, device="cuda") < 0.5] = low
    x[:, 0] = 1.0 / scale
    o = tk.logp(x, tokens, scale=scale)
    l, H, _, _ = plain.logp(x, tokens, scale)
    near(o.logp, l.float(), tol_logp(V, l))  # (-1e47 is -inf in 32 bits)
    near(o.entropy, H, rel_of(V) * (1 + math.log(V)) + 2.0 ** -22 * (math.log(V) + 1))
    dl, dh = torch.randn(161, generator=g, device="cuda"), torch.randn(161, generator=g, device="cuda")
    got = tk.logp_backward(x, tokens, o.norm, dl, entropy=o.entropy, dentropy=dh, scale=scale)
    want = plain.dlogits(x, tokens, dl, dh, scale)
    near(got, want, rel_of(V) * scale * (dl.abs() + dh.abs() * (2 + math.log(V))).double()[:, None])
    adv = torch.randn(161, generator=g, device="cuda")
    both = tk.policy_grad(tk.policy_objective(entropy_coef=0.3, mean="fixed"), x, tokens, None, adv, scale=scale)
    want = plain.dlogits(x, tokens, -adv, torch.full_like(adv, -0.3), scale)
    near(both.dlogits, want, (2.0 ** -20 + rel_of(V)) * scale * (adv.abs() + 0.3 * (2 + math.log(V))).double()[:, None])


@pytest.mark.parametrize("z", [5.0, 20.0, 30.0, 38.0, 60.0, 85.0, -85.0])
def test_preference_gradients_of_decided_pairs(tk, z):
    """The sigmoid's slope keeps its digits where it is small: terms in 64 bits, rounded once."""
    l = torch.tensor([z, 0.0], device="cuda")
    off = torch.tensor([0, 1, 2], device="cuda")
    o = tk.preference_loss(tk.preference_objective("sigmoid", beta=1.0), l, off)
    want = -1.0 / (1.0 + math.exp(z))
    assert abs(o.dlogp[0].item() - want) <= 2.0 ** -23 * abs(want) and o.dlogp[1].item() == -o.dlogp[0].item()


@pytest.mark.parametrize("R,V,dtype", [(3, 262144, "f32"), (70, 230001, "f32"), (5, 500001, "bf16"), (700, 223300, "f32")])
def test_policy_grad_of_rows_that_no_cluster_holds(tk, R, V, dtype):
    x, tokens, g = make(R, V, DT[dtype], R, ignored=0.2 if R > 3 else 0.0)
    got = check_fused(tk, x, tokens, 0.9, g)
    again = tk.policy_grad(tk.policy_objective(), x, tokens, None, torch.ones(R, device="cuda"), scale=0.9)
    assert torch.equal(again.logp, got.logp)
    obj, adv = tk.policy_objective(entropy_coef=0.1), torch.randn(R, generator=g, device="cuda")
    a = tk.policy_grad(obj, x, tokens, None, adv)
    y = x.clone()
    b = tk.policy_grad(obj, y, tokens, None, adv, out=y)  # in place
    assert torch.equal(y, a.dlogits) and torch.equal(a.stats, b.stats)


@pytest.mark.parametrize("R,V,dtype", [(14500, 1500, "bf16"), (9100, 5000, "bf16"), (9100, 2500, "f32"), (3500, 15000, "bf16"), (1500, 60000, "bf16"), (1500, 40000, "f32"), (480, 220000, "f16")])
def test_a_dozen_rows_a_cluster(tk, R, V, dtype):
    """Rows held on chip, so many that every block or cluster takes a dozen: sets of sums and constants are used again, with rows that do not count
    between those that do, one at a time and many in a row."""
    x, tokens, g = make(R, V, DT[dtype], R, ignored=0.3)
    tokens[R // 3: R // 2] = -100
    x[tokens < 0] = math.nan
    S = 9
    _, _, adv, _, _, offsets, _ = policy_inputs(R, S, g, R // 20)
    f, obj = objective(tk, mean="sequence", kl="k2")
    step = max(1, (1 << 26) // V)  # (64-bit forms of a few rows at a time)
    parts = [plain.logp(x[r: r + step], tokens[r: r + step])[:2] for r in range(0, R, step)]
    l, H = (torch.cat([p[i] for p in parts]) for i in (0, 1))
    old = off_the_edge(f, l, (l + 0.2 * torch.randn(R, generator=g, device="cuda")).float())
    ref = (l + 0.2 * torch.randn(R, generator=g, device="cuda")).float()
    got = tk.policy_grad(obj, x, tokens, old, adv, ref_logp=ref, offsets=offsets)
    stats, dl, dh = plain.policy(f, l, old, adv, ref, H, tokens, None, offsets)
    near(got.logp, l, tol_logp(V, l))
    near(got.entropy, H, rel_of(V) * (1 + math.log(V)) + 2.0 ** -22 * (math.log(V) + 1))
    near(got.stats, stats, (2.0 ** -19 + 4 * float(tol_logp(V, l).max())) * (2 + float(adv.abs().max()) + math.log(V)))
    slack = (2.0 ** -20 + 3 * tol_logp(V, l) + rel_of(V)) * (dl.abs() + dh.abs() * (2 + math.log(V)) + dl.abs().max())
    for r in range(0, R, step):
        at = slice(r, r + step)
        want = plain.dlogits(x[at], tokens[at], dl[at], dh[at])
        near(got.dlogits[at], want, half(x.dtype) * want.abs() + tiny(x.dtype) + slack[at, None])
    o = tk.logp(x[:590], tokens[:590])  # (so many rows of the longer ones go through clusters in this call, too)
    near(o.logp, l[:590], tol_logp(V, l[:590]))
    near(o.entropy, H[:590], rel_of(V) * (1 + math.log(V)) + 2.0 ** -22 * (math.log(V) + 1))


@pytest.mark.parametrize("R,V,dtype,scale,most", [(8000, 300, torch.float32, 1.0, 1.2e-8), (8000, 300, torch.float32, 0.7, 1.2e-8),
                                                  (2000, 9823, torch.float16, 0.7, 6.5e-8), (2000, 40000, torch.bfloat16, 0.7, 9.4e-8)])
def test_what_the_roundings_have_in_common_is_taken_out(tk, R, V, dtype, scale, most):
    """The mean error of log p over 10 R rows.  Measured with the corrections 3e-9, 4e-9, 5.1e-8 and 7.3e-8, without them 1.5e-8, 3.8e-8, 8.2e-8 and 1.14e-7:
    the bounds lie between, five deviations of the mean (rows deviate by 3.5e-7 at most: 6e-9 and 1.25e-8) off either."""
    s32 = torch.tensor(scale, dtype=torch.float32).double().item()
    errs = []
    for seed in range(10):
        x, tokens, _ = make(R, V, dtype, 100 + seed)
        errs.append(tk.logp(x, tokens, scale).logp.double() - plain.logp(x, tokens, s32)[0])
    err = torch.cat(errs)
    assert abs(err.mean().item()) < most, err.mean().item()
