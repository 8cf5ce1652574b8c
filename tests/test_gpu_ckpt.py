"""Activation checkpoints in 8 bits on the GPU against the format in 64 bits, and the gradients that are taken from them."""
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


def matrix(R, K, dtype, seed=0, pad=0, shift=0, sd=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((shift + R * (K + pad) + 8,), math.nan, dtype=dtype, device="cuda")
    x = flat[shift: shift + R * (K + pad)].view(R, K + pad)[:, :K]
    x.copy_(torch.randn(R, K, generator=g, device="cuda") * torch.exp(2 * torch.randn(1, K, generator=g, device="cuda")) * sd)
    return x


def near(got, want, tol):
    got, want = got.double(), want.double()
    same = (got == want) | (got.isnan() & want.isnan())
    tol = torch.as_tensor(tol, dtype=torch.float64, device=got.device).expand_as(want)
    bad = ~same & ~((got - want).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, the first at {bad.nonzero()[0].tolist()}: {got[bad][0].item()} for {want[bad][0].item()}, tolerance {tol[bad][0].item()}"


def half(dtype):
    return torch.finfo(dtype).eps / 2


SHAPES = [(1, 1, 0, 0), (3, 5, 0, 0), (64, 64, 0, 0), (7, 31, 1, 1), (33, 33, 0, 0), (5, 100, 4, 0), (129, 257, 7, 3), (2, 5000, 0, 0), (4097, 96, 0, 0)]


@pytest.mark.parametrize("act", ["identity", "relu", "silu", "gelu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,K,pad,shift", SHAPES)
def test_forward_and_backward(tk, R, K, pad, shift, dtype, act):
    """The kept values are exact (one rounding, ties to even).  act(x): sums and quotients of a few fp32 operations, 2^-20 of the largest term, then
    one rounding to the type."""
    dt = DT[dtype]
    x = matrix(R, K, dt, R + K, pad, shift)
    y, ck = tk.ckpt_forward(x, act)
    want, E = plain.kept(x)
    assert torch.equal(ck.scales.long(), E + 127)
    assert (ck.codes[:, K:] == 0).all()
    assert torch.equal(tk.ckpt_unpack(ck, torch.float32).double(), want)
    lim = torch.finfo(dt).max
    assert torch.equal(tk.ckpt_unpack(ck, dt), want.clamp(-lim, lim).to(dt))
    tiny = torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
    fx = plain.act(act, x.double())
    near(y, fx, half(dt) * fx.abs() + tiny + (2.0 ** -20 * x.double().abs() if act in ("silu", "gelu") else 0.0))
    dy = matrix(R, K, dt, 7, pad, shift, 1e-2)
    dx = tk.ckpt_backward(ck, dy, act)
    s = plain.slope(act, want)
    ref = dy.double() * s
    near(dx, ref, half(dt) * ref.abs() + tiny + (2.0 ** -20 * dy.double().abs() * (1 + want.abs().clamp(max=20)) if act in ("silu", "gelu") else 2.0 ** -24 * ref.abs()))
    # without y, and in place
    none, again = tk.ckpt_forward(x, act, y=False)
    assert none is None and torch.equal(again.codes, ck.codes) and torch.equal(again.scales, ck.scales)
    tk.ckpt_backward(ck, dy, act, out=dy)
    assert torch.equal(dy, dx)
    tk.ckpt_forward(x, act, out=x)
    assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_every_value_of_the_type_that_fits(tk, dtype):
    """Blocks around one number: all 16-bit numbers of the type (for fp32: those of bf16, and random bits)."""
    dt = DT[dtype]
    bits = torch.arange(1 << 16, device="cuda").to(torch.int32)
    if dtype == "f32":
        g = torch.Generator(device="cuda").manual_seed(0)
        v = torch.cat(((bits << 16).view(torch.float32), torch.randint(-(1 << 31), 1 << 31, (1 << 16,), generator=g, device="cuda", dtype=torch.int64).to(torch.int32).view(torch.float32)))
    else:
        v = (bits - (1 << 15)).to(torch.int16).view(dt)
    x = v.view(-1, 32).contiguous()
    _, ck = tk.ckpt_forward(x, "identity")
    want, E = plain.kept(x)
    got = tk.ckpt_unpack(ck, torch.float32).double()
    assert torch.equal(ck.scales.long(), E + 127)
    assert torch.equal(got.nan_to_num(nan=-12345.0), want.nan_to_num(nan=-12345.0))
    one = v.view(-1, 1).contiguous()  # each number alone in its block
    _, ck = tk.ckpt_forward(one, "identity")
    got = tk.ckpt_unpack(ck, torch.float32).double()
    ok = one.isfinite()
    assert got[~ok].isnan().all()
    # 2^-4 of the value, down to where the smallest scale ends: half of 2^-9 2^-117
    near(got[ok], one[ok].double(), 2.0 ** -4 * one[ok].double().abs() + 2.0 ** -127)


def test_ties_and_specials(tk):
    x = torch.zeros(6, 32, device="cuda")
    x[0, 0] = 448.0
    x[0, 1:9] = torch.tensor([17.0, 19.0, 21.0, -17.0, 232.0, 2.0 ** -10, 3 * 2.0 ** -10, 440.0])  # ties: to even
    x[1, 0], x[1, 1] = 449.0, 1.0  # one power of two up
    x[2] = torch.nan
    x[3, 3], x[3, 4], x[3, 5] = math.inf, -math.inf, 2.0
    x[4] = 3.4028234663852886e38
    x[5, 0] = 1e-45
    y, ck = tk.ckpt_forward(x, "relu")
    got = tk.ckpt_unpack(ck, torch.float32)
    assert got[0, :9].tolist() == [448.0, 16.0, 20.0, 20.0, -16.0, 224.0, 0.0, 2.0 ** -8, 448.0]
    assert ck.scales[0, 0] == 127 and ck.scales[1, 0] == 128 and ck.scales[2, 0] == 10
    assert got[2].isnan().all() and got[3, 3:5].isnan().all() and got[3, 5] == 2.0 and (got[3, 6:] == 0).all()
    assert got[4].isfinite().all() and (got[4] == 240 * 2.0 ** 120).all() and (got[5] == 0).all()
    assert y[2].isnan().all() and y[3, 3] == math.inf and y[3, 4] == 0


def test_every_nan_is_one_code(tk):
    """Whatever its sign: ReLU's gradient by sign bits must not lose it."""
    for dt in DT.values():
        x = torch.zeros(2, 32, dtype=dt, device="cuda")
        x[0, 5], x[1, 6] = math.nan, -math.nan
        x[1, 6] = torch.copysign(torch.tensor(math.nan), torch.tensor(-1.0)).to(dt)
        _, ck = tk.ckpt_forward(x, "identity")
        assert ck.codes[0, 5] == 0x7F and ck.codes[1, 6] == 0x7F and (ck.codes != 0).sum() == 2
        assert tk.ckpt_weight_grad(ck, torch.ones(2, 3, device="cuda"), "relu")[[5, 6]].isnan().all()
        dx = tk.ckpt_backward(ck, torch.ones_like(x), "relu")
        assert dx[0, 5].isnan() and dx[1, 6].isnan() and dx.isnan().sum() == 2


def test_no_rows(tk):
    x = torch.empty(0, 40, device="cuda")
    y, ck = tk.ckpt_forward(x, "silu")
    assert y.shape == (0, 40) and tk.ckpt_unpack(ck).shape == (0, 40) and tk.ckpt_backward(ck, x, "silu").shape == (0, 40)


def wgrad_want(ck, dy, act, tk):
    x = tk.ckpt_unpack(ck, torch.float32).double()
    return plain.act(act, x).t() @ dy.double(), plain.act(act, x).abs().t() @ dy.double().abs()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,K,N,pad", [(1, 1, 1, 0), (1, 33, 70, 0), (5, 64, 8, 0), (63, 32, 64, 0), (64, 128, 65, 7), (65, 129, 128, 8), (1000, 200, 129, 0), (513, 96, 256, 0),
                                       (2049, 40, 257, 3), (5000, 300, 520, 8), (40000, 64, 64, 0), (300, 1030, 1000, 0), (129, 257, 263, 7), (5003, 300, 4099, 0),
                                       (2600, 512, 2048, 0), (30000, 260, 72, 1), (32, 65, 129, 1), (17, 160, 300, 0), (33, 500, 700, 0),
                                       (2048, 64, 130, 3), (2049, 1, 1, 0), (3000, 33, 70, 0), (2113, 128, 65, 7), (2500, 129, 128, 8), (4100, 200, 129, 0), (50, 2100, 777, 0)])
def test_weight_grad(tk, R, K, N, pad, dtype):
    """Products are exact; the sums: up to 32 accumulations toward zero in an accumulator (2^-23 of its size each), then one addition a group of 512
    rows at most and one a split (2^-24 each): 2^-23 (32 + R/128) of the sum of the absolute values is a bound.  (Small ones: 32 roundings of 2^-24 and one for each 16 rows.)"""
    dt = DT[dtype]
    x = matrix(R, K, torch.float32, R + K, sd=0.3)
    _, ck = tk.ckpt_forward(x, "relu")
    dy = matrix(R, N, dt, N, pad, 1 if pad == 7 else 0, 1e-2)
    for act in ("identity", "relu"):
        want, size = wgrad_want(ck, dy, act, tk)
        tol = 2.0 ** -23 * (32 + R / 128) * size + 1e-30
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = tk.ckpt_weight_grad(ck, dy, act, status=status)
        near(got, want, tol)
        assert status.item() == 0
        assert torch.equal(got, tk.ckpt_weight_grad(ck, dy, act))
        wide = torch.full((K, N + 5), 3.0, device="cuda")
        tk.ckpt_weight_grad(ck, dy, act, out=wide[:, :N], accumulate=True)
        near(wide[:, :N], want + 3.0, tol + 2.0 ** -22 * (3.0 + want.abs()))
        assert (wide[:, N:] == 3).all()
        tk.ckpt_weight_grad(ck, dy, act, out=wide[:, :N])
        assert torch.equal(wide[:, :N], got) and (wide[:, N:] == 3).all()


def test_weight_grad_has_the_accuracy_of_its_operands(tk):
    """Long sums of one sign, where a bias would add up."""
    R = 200000
    x = torch.rand(R, 32, device="cuda") + 0.5
    _, ck = tk.ckpt_forward(x, "identity")
    for dt in (torch.float32, torch.bfloat16):
        dy = (torch.rand(R, 16, device="cuda") + 0.5).to(dt)
        want, _ = wgrad_want(ck, dy, "identity", tk)
        rel = (tk.ckpt_weight_grad(ck, dy).double() / want - 1).abs().max().item()
        assert rel < 4e-6, rel


def test_weight_grad_corners(tk):
    e = tk.Checkpoint(torch.empty(0, 64, dtype=torch.uint8, device="cuda"), torch.empty(0, 2, dtype=torch.uint8, device="cuda"), 40)
    got = tk.ckpt_weight_grad(e, torch.empty(0, 7, device="cuda"))
    assert got.shape == (40, 7) and (got == 0).all()
    acc = torch.ones(40, 7, device="cuda")
    tk.ckpt_weight_grad(e, torch.empty(0, 7, device="cuda"), out=acc, accumulate=True)
    assert (acc == 1).all()
    # values that are not numbers stay in their row of dW, or column
    x = torch.ones(70, 40, device="cuda")
    x[3, 7] = math.nan
    _, ck = tk.ckpt_forward(x, "identity")
    dy = torch.ones(70, 20, device="cuda")
    dy[5, 2] = math.inf
    dy[6, 4] = 3.4e38
    got = tk.ckpt_weight_grad(ck, dy)
    assert got[7].isnan().all() and (got[:7, 2] == math.inf).all() and (got[8:, 2] == math.inf).all()
    keep = torch.ones(20, dtype=torch.bool, device="cuda")
    keep[2] = False
    assert got[:7][:, keep].isfinite().all() and (got[0, 0] == 70) and (got[0, 4].item() / 3.4e38 - 1) < 1e-6
    for dt in (torch.bfloat16, torch.float16):
        assert (tk.ckpt_weight_grad(ck, torch.ones(70, 20, dtype=dt, device="cuda"))[0] == 70).all()


def test_a_layer_and_a_policy_together(tk):
    """A hidden layer kept in 8 bits, a vocabulary of logits, the clipped loss with its gradient, the weights' gradients from the checkpoint:
    captured into one graph, against 64-bit formulas on the values that the kernels were given."""
    R, D, K, V = 700, 48, 96, 1003
    g = torch.Generator(device="cuda").manual_seed(9)
    inp = torch.randn(R, D, generator=g, device="cuda")
    W1 = torch.randn(D, K, generator=g, device="cuda") / D ** 0.5
    W2 = torch.randn(K, V, generator=g, device="cuda") / K ** 0.5
    tokens = torch.randint(0, V, (R,), generator=g, device="cuda")
    tokens[::7] = -100
    offsets = torch.tensor([0, 100, 100, 350, 690], device="cuda")
    adv = torch.randn(R, generator=g, device="cuda")
    f = dict(clip_low=0.2, clip_high=0.2, dual_clip=0.0, kl="k3", kl_coef=0.1, entropy_coef=0.02, mean="sequence", divisor=1.0)
    obj = tk.policy_objective(**f)
    logits0 = torch.relu(inp @ W1) @ W2
    l0 = tk.logp(logits0, tokens).logp
    ref = l0 + 0.1 * torch.randn(R, generator=g, device="cuda")

    def step():
        _, inp_ck = tk.ckpt_forward(inp, "identity", y=False)
        h = inp @ W1
        y, ck = tk.ckpt_forward(h, "relu")
        logits = y @ W2
        o = tk.policy_grad(obj, logits, tokens, None, adv, ref_logp=ref, offsets=offsets)
        dW2 = tk.ckpt_weight_grad(ck, o.dlogits, "relu")
        dy = o.dlogits @ W2.t()
        dh = tk.ckpt_backward(ck, dy, "relu")
        return h, logits, o, dW2, dy, dh, tk.ckpt_weight_grad(inp_ck, dh)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h, logits, o, dW2, dy, dh, dW1 = step()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    lp, H, _, _ = plain.logp(logits, tokens)
    stats, dl, dent = plain.policy(f, lp, None, adv, ref, H, tokens, None, offsets)
    near(o.stats, stats, 1e-4)
    want = plain.dlogits(logits, tokens, dl, dent)
    near(o.dlogits, want, 1e-5 * want.abs().max())
    hq, iq = plain.kept(h)[0], plain.kept(inp)[0]
    w2 = plain.act("relu", hq).t() @ o.dlogits.double()
    near(dW2, w2, 2.0 ** -23 * 40 * (plain.act("relu", hq).t() @ o.dlogits.double().abs()) + 1e-30)
    assert torch.equal(dh, torch.where(hq > 0, dy, torch.zeros_like(dy)))  # (dy itself is torch's product, off by its own sums)
    near(dW1, iq.t() @ dh.double(), 2.0 ** -23 * 40 * (iq.abs().t() @ dh.double().abs()) + 1e-30)
    # against the gradient of a layer that was kept whole: the 8 bits' 2^-4 an element, averaged over hundreds of rows
    full = torch.relu(h).double().t() @ o.dlogits.double()
    assert (dW2.double() - full).norm() / full.norm() < 2.0 ** -4


def test_matrices_past_32_bits(tk):
    R, K = 70000, 65536  # 4.6e9 elements
    x = torch.zeros(R, K, dtype=torch.bfloat16, device="cuda")
    x[-1] = torch.arange(K, device="cuda") % 13 - 6
    y, ck = tk.ckpt_forward(x, "relu", out=x)
    assert torch.equal(tk.ckpt_unpack(tk.Checkpoint(ck.codes[-1:], ck.scales[-1:], K))[0], (torch.arange(K, device="cuda") % 13 - 6).float())
    assert (ck.codes[:-1:997] == 0).all() and torch.equal(x[-1].float(), (torch.arange(K, device="cuda") % 13 - 6).clamp(min=0).float())
    x.fill_(1.0)
    tk.ckpt_backward(ck, x, "relu", out=x)
    assert torch.equal(x[-1], (torch.arange(K, device="cuda") % 13 > 6).to(torch.bfloat16)) and (x[-2] == 0).all()


def test_refusals_of_tensors(tk):
    """Types, shapes, strides and devices that do not fit; nothing is enqueued and the next call is sound."""
    x = torch.randn(6, 40, device="cuda")
    y, ck = tk.ckpt_forward(x)
    dy = torch.randn(6, 8, device="cuda")
    q, s, _ = ck
    Ck = tk.Checkpoint
    bad = [Ck(q, s, 0), Ck(q, s, -3), Ck(q, s, 70), Ck(q, s, 32), Ck(q, s, 1 << 40), Ck(q[:, :40], s, 40), Ck(q.int(), s, 40), Ck(q.cpu(), s.cpu(), 40), Ck(q, s.cpu(), 40),
           Ck(q, s[:5], 40), Ck(q, s.t().contiguous().t(), 40), Ck(q[:5], s, 40), Ck(None, s, 40), Ck(q, None, 40)]
    calls = [lambda f=f, c=c: f(c) for c in bad for f in (tk.ckpt_unpack, lambda c: tk.ckpt_backward(c, x), lambda c: tk.ckpt_weight_grad(c, dy))]
    calls += [lambda: tk.ckpt_forward(x.double()), lambda: tk.ckpt_forward(x.t()), lambda: tk.ckpt_forward(x, "tanh"), lambda: tk.ckpt_forward(x, out=x.half()),
              lambda: tk.ckpt_forward(x, out=x[:5]), lambda: tk.ckpt_unpack(ck, torch.float64), lambda: tk.ckpt_unpack(ck, out=x.double()), lambda: tk.ckpt_unpack(ck, out=x[:, 1:]),
              lambda: tk.ckpt_backward(ck, x[:5]), lambda: tk.ckpt_backward(ck, None), lambda: tk.ckpt_backward(ck, x.cpu()), lambda: tk.ckpt_backward(ck, x, "tanh"),
              lambda: tk.ckpt_backward(ck, x, out=x.half()), lambda: tk.ckpt_weight_grad(ck, dy[:5]), lambda: tk.ckpt_weight_grad(ck, dy, accumulate=True),
              lambda: tk.ckpt_weight_grad(ck, dy, out=torch.zeros(40, 8, device="cuda").half()), lambda: tk.ckpt_weight_grad(ck, dy, out=torch.zeros(8, 40, device="cuda")),
              lambda: tk.ckpt_weight_grad(ck, dy, status=torch.zeros(1, device="cuda")), lambda: tk.ckpt_weight_grad(ck, dy, status=torch.zeros(2, dtype=torch.int32, device="cuda"))]
    for i, call in enumerate(calls):
        with pytest.raises(tk.AnakinError) as e:
            call()
            print(f"call {i} was taken")
        assert e.value.code == -1, i
    for act in ("silu", "gelu"):
        with pytest.raises(tk.AnakinError) as e:
            tk.ckpt_weight_grad(ck, dy, act)
        assert e.value.code == -4
    again = tk.ckpt_forward(x)
    assert torch.equal(again[0], y) and torch.equal(again[1].codes, q) and torch.equal(again[1].scales, s)


@pytest.mark.parametrize("act,lo,hi", [("silu", -100.0, -3.0), ("gelu", -14.0, -2.0)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_tails_of_the_activations(tk, dtype, act, lo, hi):
    """Where they are near 0, against their own size.  fp32: the exponential's 2^-22, the quotient's 2 ulp, polynomial and products: 1.1 2^-20 of the value,
    2^-19 is allowed; the slopes' two terms cancel by a factor below 2 there.  16-bit types: the fit's 7e-5 and the exponent's rounding, 2^-13 is allowed beside
    the type's own half step.  Exponentials below 2^-126 are 0."""
    dt = DT[dtype]
    x = torch.linspace(lo, hi, 96 * 64, device="cuda").view(96, 64).to(dt)
    rel = 2.0 ** -19 if dtype == "f32" else half(dt) + 2.0 ** -13
    least = 2.0 ** -118 if dtype != "f16" else torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
    y, ck = tk.ckpt_forward(x, act)
    below = lambda v: 0.5 * torch.erfc(-v / math.sqrt(2.0))  # noqa: E731  (the normal distribution function; 1 + erf would lose it here)
    v = x.double()
    want = v * torch.sigmoid(v) if act == "silu" else v * below(v)
    near(y, want, rel * want.abs() + least)
    v = plain.kept(x)[0]
    dx = tk.ckpt_backward(ck, torch.ones_like(x), act)
    want = plain.slope(act, v) if act == "silu" else below(v) + v * torch.exp(-v * v / 2) / math.sqrt(2.0 * math.pi)
    near(dx, want, rel * want.abs() + least)
