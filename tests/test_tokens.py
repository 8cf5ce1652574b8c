"""Host side of the operators over token rows and of the 8-bit checkpoints: what they refuse, sizes, and the formulas that the GPU tests compare with
(no GPU work is enqueued by anything here)."""
import ctypes as C
import math

import pytest
import torch

from tests import token_plain as plain

FAKE = C.c_void_p(0x10000)  # never read: every call below ends before it enqueues anything


@pytest.fixture(scope="module")
def tk():
    from paper_2104_06272_b200 import build

    build.build()
    from paper_2104_06272_b200 import tokens

    return tokens


def rows_of(tk, **kw):
    f = dict(struct_size=C.sizeof(tk.TokenRows), dtype=1, rows=10, vocab=100, ld=100, logits=0x10000, tokens=0x10000, token_bytes=8, scale=1.0)
    f.update(kw)
    return tk.TokenRows(**f)


def test_structs_have_the_c_layout(tk):
    assert (C.sizeof(tk.TokenRows), C.sizeof(tk.PolicyObjective), C.sizeof(tk.PreferenceObjective)) == (88, 36, 24)


@pytest.mark.parametrize("kw", [dict(struct_size=80), dict(reserved=1), dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(rows=1 << 31), dict(vocab=0),
                                dict(vocab=1 << 31), dict(ld=99), dict(logits=None), dict(logits=0x10001), dict(dtype=0, logits=0x10002), dict(tokens=None),
                                dict(tokens=0x10004), dict(token_bytes=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan),
                                dict(offsets=0x10000, offset_bytes=3), dict(offsets=0x10004, offset_bytes=8), dict(sequences=-1)])
def test_bad_rows_are_refused(tk, kw):
    r = rows_of(tk, **kw)
    lib, bad = tk._lib, -1
    obj = tk.policy_objective()
    assert lib.anakin_token_logp(C.byref(r), FAKE, FAKE, FAKE, None) == bad
    assert lib.anakin_token_logp_backward(C.byref(r), FAKE, FAKE, FAKE, FAKE, FAKE, 100, None) == bad
    assert lib.anakin_token_policy_grad(C.byref(r), C.byref(obj), FAKE, FAKE, None, FAKE, FAKE, FAKE, FAKE, 100, FAKE, 1 << 30, None) == bad


def test_missing_outputs_and_inputs_are_refused(tk):
    lib, r, bad, small = tk._lib, rows_of(tk), -1, -3
    obj, kl = tk.policy_objective(), tk.policy_objective(kl="k3", kl_coef=0.1)
    assert lib.anakin_token_logp(None, FAKE, FAKE, FAKE, None) == bad
    assert lib.anakin_token_logp(C.byref(r), None, FAKE, FAKE, None) == bad
    back = lambda norm=FAKE, H=FAKE, dl=FAKE, dh=FAKE, out=FAKE, ld=100: lib.anakin_token_logp_backward(C.byref(r), norm, H, dl, dh, out, ld, None)  # noqa: E731
    assert back(norm=None) == back(H=None) == back(dl=None) == back(out=None) == back(ld=99) == bad

    def grad(o=obj, old=FAKE, adv=FAKE, ref=None, stats=FAKE, out=FAKE, ld=100, ws=FAKE, n=1 << 30):
        return lib.anakin_token_policy_grad(C.byref(r), C.byref(o), old, adv, ref, stats, None, None, out, ld, ws, n, None)

    assert grad(adv=None) == grad(stats=None) == grad(out=None) == grad(ld=99) == grad(o=kl) == grad(ws=None) == grad(ws=C.c_void_p(0x10010)) == bad
    assert grad(n=16) == small

    def loss(o=obj, lp=FAKE, adv=FAKE, ref=None, stats=FAKE, out=FAKE, ws=FAKE, n=1 << 30):
        return lib.anakin_token_policy_loss(C.byref(r), C.byref(o), lp, None, adv, ref, None, stats, out, None, ws, n, None)

    assert loss(lp=None) == loss(adv=None) == loss(stats=None) == loss(out=None) == loss(o=kl) == loss(ws=None) == bad
    assert loss(n=16) == small
    pr = rows_of(tk, offsets=0x10000, offset_bytes=8, sequences=4)

    def pref(rows=pr, o=tk.preference_objective(), lp=FAKE, stats=FAKE, z=FAKE, out=FAKE, ws=FAKE, n=1 << 30):
        return lib.anakin_token_preference_loss(C.byref(rows), C.byref(o), lp, None, stats, z, out, ws, n, None)

    assert pref(rows=r) == pref(rows=rows_of(tk, offsets=0x10000, offset_bytes=8, sequences=3)) == bad
    assert pref(lp=None) == pref(stats=None) == pref(z=None) == pref(out=None) == pref(ws=None) == bad
    assert pref(n=16) == small


@pytest.mark.parametrize("kw", [dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_high=-0.1), dict(dual_clip=0.5), dict(dual_clip=math.nan), dict(clip_low=math.nan),
                                dict(mean="fixed", divisor=0.0), dict(mean="fixed", divisor=-1.0), dict(kl_coef=math.nan), dict(entropy_coef=math.nan)])
def test_bad_policy_objectives_are_refused(tk, kw):
    r, o = rows_of(tk), tk.policy_objective(**kw)
    assert tk._lib.anakin_token_policy_loss(C.byref(r), C.byref(o), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 30, None) == -1
    assert tk._lib.anakin_token_policy_grad(C.byref(r), C.byref(o), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 100, FAKE, 1 << 30, None) == -1


@pytest.mark.parametrize("kw", [dict(beta=0.0), dict(beta=-1.0), dict(beta=math.inf), dict(margin=math.nan), dict(smoothing=-0.1), dict(smoothing=0.6)])
def test_bad_preference_objectives_are_refused(tk, kw):
    r, o = rows_of(tk, offsets=0x10000, offset_bytes=8, sequences=4), tk.preference_objective(**kw)
    assert tk._lib.anakin_token_preference_loss(C.byref(r), C.byref(o), FAKE, None, FAKE, FAKE, FAKE, FAKE, 1 << 30, None) == -1


def test_objectives_of_unknown_names_are_refused(tk):
    for make in (lambda: tk.policy_objective(kl="k4"), lambda: tk.policy_objective(mean="all"), lambda: tk.preference_objective("other")):
        with pytest.raises(tk.AnakinError) as e:
            make()
        assert e.value.code == -1


def test_checkpoint_refusals(tk):
    lib, bad = tk._lib, -1
    n, m = C.c_size_t(0), C.c_size_t(0)
    assert lib.anakin_ckpt_bytes(10, 33, C.byref(n), C.byref(m)) == 0 and (n.value, m.value) == (640, 20)
    assert lib.anakin_ckpt_bytes(0, 1, C.byref(n), C.byref(m)) == 0 and (n.value, m.value) == (0, 0)
    assert lib.anakin_ckpt_bytes(-1, 33, C.byref(n), C.byref(m)) == lib.anakin_ckpt_bytes(1, 0, C.byref(n), C.byref(m)) == lib.anakin_ckpt_bytes(1, 1, None, C.byref(m)) == bad

    def fwd(dt=1, act=1, r=4, c=40, x=FAKE, ldx=40, y=FAKE, ldy=40, q=FAKE, s=FAKE):
        return lib.anakin_ckpt_forward(dt, act, r, c, x, ldx, y, ldy, q, s, None)

    assert fwd(dt=3) == fwd(act=4) == fwd(act=-1) == fwd(r=-1) == fwd(c=0) == fwd(x=None) == fwd(ldx=39) == fwd(ldy=39) == fwd(q=None) == fwd(s=None) == bad
    assert fwd(x=C.c_void_p(0x10001)) == fwd(q=C.c_void_p(0x10008)) == fwd(dt=0, y=C.c_void_p(0x10002)) == bad
    assert lib.anakin_ckpt_unpack(1, 4, 40, FAKE, FAKE, None, 40, None) == lib.anakin_ckpt_unpack(1, 4, 40, FAKE, FAKE, FAKE, 39, None) == bad
    assert lib.anakin_ckpt_backward(1, 1, 4, 40, FAKE, FAKE, None, 40, FAKE, 40, None) == lib.anakin_ckpt_backward(1, 7, 4, 40, FAKE, FAKE, FAKE, 40, FAKE, 40, None) == bad

    def wg(dt=1, act=1, r=4, c=40, k=8, q=FAKE, s=FAKE, dy=FAKE, ld=8, dw=FAKE, lddw=8, ws=FAKE, b=1 << 30):
        return lib.anakin_ckpt_weight_grad(dt, act, r, c, k, q, s, dy, ld, dw, lddw, 0, ws, b, None, None)

    assert wg(dt=5) == wg(act=9) == wg(r=-1) == wg(c=0) == wg(k=0) == wg(q=None) == wg(dy=None) == wg(ld=7) == wg(dw=None) == wg(lddw=7) == wg(ws=None) == bad
    assert wg(dw=C.c_void_p(0x10002)) == wg(dy=C.c_void_p(0x10001)) == wg(ws=C.c_void_p(0x10010)) == wg(k=1 << 23) == bad
    assert wg(act=2) == wg(act=3) == -4 and wg(dt=0, r=4096, b=0) == -3
    assert lib.anakin_ckpt_weight_grad_workspace_bytes(1, 4, 40, 8, 1, None) == bad


def test_host_tensors_are_refused(tk):
    x, t, v = torch.zeros(3, 5), torch.zeros(3, dtype=torch.int64), torch.zeros(3)
    obj = tk.policy_objective()
    ck = tk.Checkpoint(torch.zeros(3, 32, dtype=torch.uint8), torch.zeros(3, 1, dtype=torch.uint8), 5)
    for call in (lambda: tk.logp(x, t), lambda: tk.logp_backward(x, t, v, v), lambda: tk.policy_loss(obj, v, v, v), lambda: tk.policy_grad(obj, x, t, v, v),
                 lambda: tk.preference_loss(tk.preference_objective(), v, t), lambda: tk.ckpt_forward(x), lambda: tk.ckpt_unpack(ck), lambda: tk.ckpt_backward(ck, x),
                 lambda: tk.ckpt_weight_grad(ck, x)):
        with pytest.raises(tk.AnakinError) as e:
            call()
        assert e.value.code == -1


def test_plain_forms_are_their_own_derivatives():
    """The formulas that the GPU tests compare with, against torch's automatic differentiation."""
    g = torch.Generator().manual_seed(0)
    R, V = 30, 11
    x = torch.randn(R, V, generator=g, dtype=torch.float64, requires_grad=True)
    tokens = torch.randint(0, V, (R,), generator=g)
    tokens[::6] = -1
    old, ref, adv = (torch.randn(R, generator=g, dtype=torch.float64) for _ in range(3))
    old, ref = old * 0.2 - 2.5, ref * 0.2 - 2.5
    offsets = torch.tensor([0, 9, 9, 20, 28])
    for mean in ("token", "sequence", "fixed"):
        for kl in ("none", "k1", "k2", "k3"):
            f = dict(clip_low=0.2, clip_high=0.3, dual_clip=2.0, kl=kl, kl_coef=0.3, entropy_coef=0.1, mean=mean, divisor=7.0)
            ok, seq = plain.counted_rows(R, tokens, None, offsets)
            lp = torch.log_softmax(0.8 * x, 1)
            l = lp.gather(1, tokens.clamp(min=0)[:, None])[:, 0]
            H = -(lp.exp() * lp).sum(1)
            r = (l - old).exp()
            pg = -torch.minimum(r * adv, r.clamp(0.8, 1.3) * adv)
            pg = torch.where(adv < 0, torch.minimum(pg, -2.0 * adv), pg)
            z = l - ref
            k = {"none": 0 * z, "k1": z, "k2": z * z / 2, "k3": torch.exp(-z) - 1 + z}[kl]
            n = torch.bincount(seq[ok], minlength=4)
            w = {"token": ok.double() / ok.sum(), "sequence": ok.double() / (n[seq.clamp(0, 3)].clamp(min=1) * (n > 0).sum()), "fixed": ok.double() / 7.0}[mean]
            loss = (w * (pg + (0.3 if kl != "none" else 0.0) * k - 0.1 * H)).sum()
            want = torch.autograd.grad(loss, x)[0]
            pl, pH, _, _ = plain.logp(x.detach(), tokens, 0.8)
            stats, dl, dh = plain.policy(f, pl, old, adv, ref, pH, tokens, None, offsets)
            got = plain.dlogits(x.detach(), tokens, dl, dh, 0.8)
            assert abs(stats[0].item() - loss.item()) < 1e-12 and (got - want).abs().max() < 1e-12
    for name in ("relu", "silu", "gelu", "identity"):
        v = torch.randn(50, generator=g, dtype=torch.float64, requires_grad=True)
        assert (torch.autograd.grad(plain.act(name, v).sum(), v)[0] - plain.slope(name, v.detach())).abs().max() < 1e-12


def test_kept_values_are_the_nearest():
    """Against torch's own e4m3 conversion."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn(40, 64, generator=g) * torch.exp(4 * torch.randn(40, 1, generator=g))
    got, E = plain.kept(x)
    s = torch.exp2(E.double()).repeat_interleave(32, 1)
    want = (x.double() / s).float().to(torch.float8_e4m3fn).double() * s
    assert torch.equal(got, want)
    top = x.view(40, 2, 32).abs().amax(2).double()
    assert (top <= 448 * torch.exp2(E.double())).all() and (top > 224 * torch.exp2(E.double())).all()


def test_gradients_at_odd_addresses_are_refused(tk):
    """As the logits are: an element's address is a multiple of its size."""
    lib, obj = tk._lib, tk.policy_objective()
    for dtype, at in ((0, 0x10002), (1, 0x10001), (2, 0x10003)):
        r, out = rows_of(tk, dtype=dtype), C.c_void_p(at)
        assert lib.anakin_token_logp_backward(C.byref(r), FAKE, FAKE, FAKE, FAKE, out, 100, None) == -1
        assert lib.anakin_token_policy_grad(C.byref(r), C.byref(obj), FAKE, FAKE, None, FAKE, None, None, out, 100, FAKE, 1 << 30, None) == -1


def test_a_workspace_for_sequences_does_for_rows_without_offsets(tk):
    """Without offsets all rows are one sequence, whatever the number of sequences says: the workspace asked for with that number has room."""
    lib, n = tk._lib, C.c_size_t(0)

    def size(rows, sequences):
        assert lib.anakin_token_workspace_bytes(rows, sequences, C.byref(n)) == 0
        return n.value

    for rows in (1, 1000, 62464, 63000, 127 * 1024, 10 ** 6, (1 << 31) - 1):
        for sequences in (0, 1, 2, 3, 7, 60, 1000):
            assert size(rows, sequences) >= size(rows, 1)
