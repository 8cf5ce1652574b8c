"""Policies over token vocabularies, and activation checkpoints in 8 bits: Python functions over the stateless calls of include/anakin.h
(anakin_token_*, anakin_ckpt_*), which say what each computes.

Argument marshalling only.  Tensors lie on one CUDA device; work is enqueued on that device's current torch stream, outputs and
workspaces come from torch's allocator on that stream, nothing synchronises, and every call may be captured into a CUDA graph.  Gradients
are outputs (`logits.backward(dlogits)` hands one to autograd); the inputs are not differentiated through.  What a call refuses it
refuses with AnakinError before anything is enqueued.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple

import torch

from .binding import E_INVALID_ARG, E_UNSUPPORTED_CFG, OK, AnakinError, lib

_vp, _i64, _fp = C.c_void_p, C.c_int64, C.c_float
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTS = {"identity": 0, "relu": 1, "silu": 2, "gelu": 3}
KLS = {"none": 0, "k1": 1, "k2": 2, "k3": 3}
MEANS = {"token": 0, "sequence": 1, "fixed": 2}
PREFERENCES = {"sigmoid": 0, "hinge": 1, "squared": 2}
POLICY_STATS = ("loss", "policy", "kl", "entropy", "cut", "old_minus_new")
PREFERENCE_STATS = ("loss", "accuracy", "preferred", "other", "margin")


class TokenRows(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("rows", _i64), ("vocab", _i64), ("ld", _i64), ("logits", _vp), ("tokens", _vp),
                ("mask", _vp), ("offsets", _vp), ("sequences", _i64), ("token_bytes", C.c_int32), ("offset_bytes", C.c_int32), ("scale", _fp),
                ("reserved", C.c_uint32)]


class PolicyObjective(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("clip_low", _fp), ("clip_high", _fp), ("dual_clip", _fp), ("kl", C.c_int32), ("kl_coef", _fp),
                ("entropy_coef", _fp), ("mean", C.c_int32), ("divisor", _fp)]


class PreferenceObjective(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("kind", C.c_int32), ("beta", _fp), ("margin", _fp), ("smoothing", _fp), ("mean", C.c_int32)]


_lib = lib()
_rows, _sz = C.POINTER(TokenRows), C.POINTER(C.c_size_t)
_lib.anakin_token_logp.argtypes = [_rows, _vp, _vp, _vp, _vp]
_lib.anakin_token_logp_backward.argtypes = [_rows, _vp, _vp, _vp, _vp, _vp, _i64, _vp]
_lib.anakin_token_workspace_bytes.argtypes = [_i64, _i64, _sz]
_lib.anakin_token_policy_loss.argtypes = [_rows, C.POINTER(PolicyObjective)] + [_vp] * 9 + [C.c_size_t, _vp]
_lib.anakin_token_policy_grad.argtypes = [_rows, C.POINTER(PolicyObjective)] + [_vp] * 7 + [_i64, _vp, C.c_size_t, _vp]
_lib.anakin_token_preference_loss.argtypes = [_rows, C.POINTER(PreferenceObjective)] + [_vp] * 6 + [C.c_size_t, _vp]
_lib.anakin_ckpt_bytes.argtypes = [_i64, _i64, _sz, _sz]
_lib.anakin_ckpt_forward.argtypes = [C.c_int, C.c_int, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _vp, _vp]
_lib.anakin_ckpt_unpack.argtypes = [C.c_int, _i64, _i64, _vp, _vp, _vp, _i64, _vp]
_lib.anakin_ckpt_backward.argtypes = [C.c_int, C.c_int, _i64, _i64, _vp, _vp, _vp, _i64, _vp, _i64, _vp]
_lib.anakin_ckpt_weight_grad_workspace_bytes.argtypes = [C.c_int, _i64, _i64, _i64, _sz]
_lib.anakin_ckpt_weight_grad.argtypes = [C.c_int, C.c_int, _i64, _i64, _i64, _vp, _vp, _vp, _i64, _vp, _i64, C.c_int, _vp, C.c_size_t, _vp, _vp]


class TokenLogp(NamedTuple):
    logp: torch.Tensor  # f32 [rows]
    entropy: torch.Tensor | None  # f32 [rows]
    norm: torch.Tensor  # f32 [rows][2], for logp_backward


class PolicyLoss(NamedTuple):
    stats: torch.Tensor  # f32, POLICY_STATS
    dlogp: torch.Tensor
    dentropy: torch.Tensor | None


class PolicyGrad(NamedTuple):
    stats: torch.Tensor  # f32, POLICY_STATS
    logp: torch.Tensor
    entropy: torch.Tensor
    dlogits: torch.Tensor


class PreferenceLoss(NamedTuple):
    stats: torch.Tensor  # f32, PREFERENCE_STATS
    margin: torch.Tensor  # f32 [pairs]
    dlogp: torch.Tensor


class Checkpoint(NamedTuple):
    codes: torch.Tensor  # uint8 [rows][cols rounded up to 32]
    scales: torch.Tensor  # uint8 [rows][blocks of 32]
    cols: int


def policy_objective(clip_low: float = 0.2, clip_high: float = 0.2, dual_clip: float = 0.0, kl: str = "none", kl_coef: float = 0.0,
                     entropy_coef: float = 0.0, mean: str = "token", divisor: float = 1.0) -> PolicyObjective:
    return PolicyObjective(C.sizeof(PolicyObjective), clip_low, clip_high, dual_clip, _one_of(KLS, "kl", kl), kl_coef, entropy_coef,
                           _one_of(MEANS, "mean", mean), divisor)


def preference_objective(kind: str = "sigmoid", beta: float = 0.1, margin: float = 0.0, smoothing: float = 0.0, mean: bool = False) -> PreferenceObjective:
    return PreferenceObjective(C.sizeof(PreferenceObjective), _one_of(PREFERENCES, "kind", kind), beta, margin, smoothing, int(mean))


def _refuse(why: str, code: int = E_INVALID_ARG):
    raise AnakinError(code, why)


def _one_of(table: dict, name: str, key: str) -> int:
    if key not in table:
        _refuse(f"{name} is one of {', '.join(table)}")
    return table[key]


def _ck(rc: int):
    if rc != OK:
        raise AnakinError(rc)


def _ptr(t: torch.Tensor | None):
    return None if t is None else _vp(t.data_ptr())


def _on(dev: torch.device, name: str, t, dtype, shape) -> torch.Tensor | None:
    """t, a dense tensor of that device, type and shape, or None."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.device != dev or tuple(t.shape) != tuple(shape) or t.dtype not in (dtype if isinstance(dtype, tuple) else (dtype,)):
        _refuse(f"{name}: a tensor of {dtype}, shape {tuple(shape)}, on {dev} is needed")
    return t if t.is_contiguous() else _refuse(f"{name} is not contiguous")


def _matrix(name: str, t, dev=None, dtype=None, shape=None) -> tuple[int, int, int]:
    """(rows, cols, elements from row to row) of a matrix whose rows are dense."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dim() != 2 or t.dtype not in DTYPES or t.shape[1] < 1:
        _refuse(f"{name}: a CUDA matrix of float32, bfloat16 or float16 with at least one column is needed")
    if (dev is not None and t.device != dev) or (dtype is not None and t.dtype != dtype) or (shape is not None and tuple(t.shape) != tuple(shape)):
        _refuse(f"{name}: {dtype} of shape {tuple(shape)} on {dev} is needed")
    rows, cols = t.shape
    if (cols > 1 and t.stride(1) != 1) or (rows > 1 and t.stride(0) < cols):
        _refuse(f"{name}: columns have to lie side by side, and rows one after the other")
    return rows, cols, (t.stride(0) if rows > 1 else cols)


class _Device:
    """Makes the tensors' device current for the call and gives its current stream."""

    def __init__(self, dev: torch.device):
        self.dev = dev
        self.guard = torch.cuda.device(dev) if dev.index != torch.cuda.current_device() else None

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return _vp(torch.cuda.current_stream(self.dev).cuda_stream)

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


_INTS, _FLAGS = (torch.int64, torch.int32), (torch.bool, torch.uint8)


def _token_rows(dev, rows, tokens, mask=None, offsets=None, logits=None, scale=1.0) -> TokenRows:
    r = TokenRows(struct_size=C.sizeof(TokenRows), rows=rows, scale=scale)
    if logits is not None:
        _, r.vocab, r.ld = _matrix("logits", logits)
        r.dtype, r.logits = DTYPES[logits.dtype], logits.data_ptr()
    if _on(dev, "tokens", tokens, _INTS, (rows,)) is not None:
        r.tokens, r.token_bytes = tokens.data_ptr(), tokens.element_size()
    if _on(dev, "mask", mask, _FLAGS, (rows,)) is not None:
        r.mask = mask.data_ptr()
    if offsets is not None:
        if not isinstance(offsets, torch.Tensor) or offsets.dim() != 1 or offsets.numel() < 1:
            _refuse("offsets: one number more than there are sequences")
        _on(dev, "offsets", offsets, _INTS, tuple(offsets.shape))
        r.offsets, r.offset_bytes, r.sequences = offsets.data_ptr(), offsets.element_size(), offsets.numel() - 1
    return r


def _workspace(dev, rows: TokenRows) -> torch.Tensor:
    n = C.c_size_t(0)
    _ck(_lib.anakin_token_workspace_bytes(rows.rows, rows.sequences, C.byref(n)))
    return torch.empty(n.value, dtype=torch.uint8, device=dev)


def _like(name: str, out, like: torch.Tensor, shape=None) -> torch.Tensor:
    if out is None:
        return torch.empty(shape or tuple(like.shape), dtype=like.dtype, device=like.device)
    _matrix(name, out, like.device, like.dtype, shape or tuple(like.shape))
    return out


def _ld(t: torch.Tensor) -> int:
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def logp(logits: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, mask: torch.Tensor | None = None, entropy: bool = True) -> TokenLogp:
    """Log-probability of every row's token under softmax(scale * logits), and the entropy (anakin_token_logp)."""
    n, _, _ = _matrix("logits", logits)
    dev = logits.device
    if tokens is None:
        _refuse("tokens are needed")
    with _Device(dev) as stream:
        rows = _token_rows(dev, n, tokens, mask, None, logits, scale)
        out = TokenLogp(torch.empty(n, device=dev), torch.empty(n, device=dev) if entropy else None, torch.empty(n, 2, device=dev))
        _ck(_lib.anakin_token_logp(C.byref(rows), _ptr(out.logp), _ptr(out.entropy), _ptr(out.norm), stream))
    return out


def logp_backward(logits: torch.Tensor, tokens: torch.Tensor, norm: torch.Tensor, dlogp: torch.Tensor, entropy: torch.Tensor | None = None,
                  dentropy: torch.Tensor | None = None, scale: float = 1.0, mask: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """Gradient of the logits from those of logp and entropy (anakin_token_logp_backward).  norm and entropy come from logp() with the same
    tokens, scale and mask; `out` may be the logits themselves."""
    n, _, _ = _matrix("logits", logits)
    dev, f32 = logits.device, torch.float32
    if tokens is None or norm is None or dlogp is None or (dentropy is not None and entropy is None):
        _refuse("tokens, norm and dlogp are needed, and entropy with dentropy")
    with _Device(dev) as stream:
        rows = _token_rows(dev, n, tokens, mask, None, logits, scale)
        _on(dev, "norm", norm, f32, (n, 2)), _on(dev, "dlogp", dlogp, f32, (n,)), _on(dev, "entropy", entropy, f32, (n,)), _on(dev, "dentropy", dentropy, f32, (n,))
        out = _like("out", out, logits)
        _ck(_lib.anakin_token_logp_backward(C.byref(rows), _ptr(norm), _ptr(entropy), _ptr(dlogp), _ptr(dentropy), _ptr(out), _ld(out), stream))
    return out


def policy_loss(objective: PolicyObjective, logp: torch.Tensor, old_logp: torch.Tensor | None, adv: torch.Tensor, ref_logp: torch.Tensor | None = None,
                entropy: torch.Tensor | None = None, mask: torch.Tensor | None = None, offsets: torch.Tensor | None = None,
                tokens: torch.Tensor | None = None) -> PolicyLoss:
    """The clipped policy loss from log-probabilities, and its gradients (anakin_token_policy_loss)."""
    if not isinstance(logp, torch.Tensor) or not logp.is_cuda or logp.dim() != 1:
        _refuse("logp: a CUDA vector is needed")
    n, dev, f32 = logp.numel(), logp.device, torch.float32
    for name, t in (("logp", logp), ("old_logp", old_logp), ("adv", adv), ("ref_logp", ref_logp), ("entropy", entropy)):
        _on(dev, name, t, f32, (n,))
    if adv is None or (objective.kl != 0 and ref_logp is None):
        _refuse("adv is needed, and ref_logp with a KL term")
    with _Device(dev) as stream:
        rows = _token_rows(dev, n, tokens, mask, offsets)
        ws = _workspace(dev, rows)
        out = PolicyLoss(torch.empty(len(POLICY_STATS), device=dev), torch.empty(n, device=dev), torch.empty(n, device=dev) if entropy is not None else None)
        _ck(_lib.anakin_token_policy_loss(C.byref(rows), C.byref(objective), _ptr(logp), _ptr(old_logp), _ptr(adv), _ptr(ref_logp), _ptr(entropy),
                                          _ptr(out.stats), _ptr(out.dlogp), _ptr(out.dentropy), _ptr(ws), ws.numel(), stream))
    return out


def policy_grad(objective: PolicyObjective, logits: torch.Tensor, tokens: torch.Tensor, old_logp: torch.Tensor | None, adv: torch.Tensor,
                ref_logp: torch.Tensor | None = None, mask: torch.Tensor | None = None, offsets: torch.Tensor | None = None, scale: float = 1.0,
                out: torch.Tensor | None = None) -> PolicyGrad:
    """The clipped policy loss from logits, with the gradient of the logits (anakin_token_policy_grad); `out` may be the logits themselves."""
    n, _, _ = _matrix("logits", logits)
    dev, f32 = logits.device, torch.float32
    for name, t in (("old_logp", old_logp), ("adv", adv), ("ref_logp", ref_logp)):
        _on(dev, name, t, f32, (n,))
    if tokens is None or adv is None or (objective.kl != 0 and ref_logp is None):
        _refuse("tokens and adv are needed, and ref_logp with a KL term")
    with _Device(dev) as stream:
        rows = _token_rows(dev, n, tokens, mask, offsets, logits, scale)
        ws = _workspace(dev, rows)
        o = PolicyGrad(torch.empty(len(POLICY_STATS), device=dev), torch.empty(n, device=dev), torch.empty(n, device=dev), _like("out", out, logits))
        _ck(_lib.anakin_token_policy_grad(C.byref(rows), C.byref(objective), _ptr(old_logp), _ptr(adv), _ptr(ref_logp), _ptr(o.stats), _ptr(o.logp),
                                          _ptr(o.entropy), _ptr(o.dlogits), _ld(o.dlogits), _ptr(ws), ws.numel(), stream))
    return o


def preference_loss(objective: PreferenceObjective, logp: torch.Tensor, offsets: torch.Tensor, ref_logp: torch.Tensor | None = None,
                    mask: torch.Tensor | None = None, tokens: torch.Tensor | None = None) -> PreferenceLoss:
    """The preference loss over pairs of sequences, the preferred ones first, and its gradient (anakin_token_preference_loss)."""
    if not isinstance(logp, torch.Tensor) or not logp.is_cuda or logp.dim() != 1:
        _refuse("logp: a CUDA vector is needed")
    n, dev = logp.numel(), logp.device
    _on(dev, "logp", logp, torch.float32, (n,)), _on(dev, "ref_logp", ref_logp, torch.float32, (n,))
    if offsets is None or not isinstance(offsets, torch.Tensor) or offsets.numel() % 2 == 0:
        _refuse("offsets of an even number of sequences are needed")
    with _Device(dev) as stream:
        rows = _token_rows(dev, n, tokens, mask, offsets)
        ws = _workspace(dev, rows)
        out = PreferenceLoss(torch.empty(len(PREFERENCE_STATS), device=dev), torch.empty(rows.sequences // 2, device=dev), torch.empty(n, device=dev))
        _ck(_lib.anakin_token_preference_loss(C.byref(rows), C.byref(objective), _ptr(logp), _ptr(ref_logp), _ptr(out.stats), _ptr(out.margin),
                                              _ptr(out.dlogp), _ptr(ws), ws.numel(), stream))
    return out


def _checkpoint(ck: Checkpoint) -> tuple[torch.device, int, int]:
    blocks = (ck.cols + 31) // 32
    if ck.cols < 1 or not isinstance(ck.codes, torch.Tensor) or not ck.codes.is_cuda or ck.codes.dim() != 2:
        _refuse("codes: a CUDA matrix of uint8 is needed")
    dev, rows = ck.codes.device, ck.codes.shape[0]
    _on(dev, "codes", ck.codes, torch.uint8, (rows, blocks * 32)), _on(dev, "scales", ck.scales, torch.uint8, (rows, blocks))
    return dev, rows, ck.cols


def ckpt_forward(x: torch.Tensor, act: str = "relu", y: bool = True, out: torch.Tensor | None = None) -> tuple[torch.Tensor | None, Checkpoint]:
    """act(x) (None with y=False) and the checkpoint of x in 8 bits (anakin_ckpt_forward); `out` may be x itself."""
    rows, cols, ld = _matrix("x", x)
    a, dev, blocks = _one_of(ACTS, "act", act), x.device, (cols + 31) // 32
    with _Device(dev) as stream:
        res = _like("out", out, x) if y else None
        ck = Checkpoint(torch.empty(rows, blocks * 32, dtype=torch.uint8, device=dev), torch.empty(rows, blocks, dtype=torch.uint8, device=dev), cols)
        _ck(_lib.anakin_ckpt_forward(DTYPES[x.dtype], a, rows, cols, _ptr(x), ld, _ptr(res), _ld(res) if y else 0, _ptr(ck.codes), _ptr(ck.scales), stream))
    return res, ck


def ckpt_unpack(ck: Checkpoint, dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None) -> torch.Tensor:
    """The values that a checkpoint holds (anakin_ckpt_unpack)."""
    dev, rows, cols = _checkpoint(ck)
    if out is not None:
        _matrix("out", out, dev, out.dtype, (rows, cols))
        dtype = out.dtype
    if dtype not in DTYPES:
        _refuse("float32, bfloat16 or float16")
    with _Device(dev) as stream:
        out = torch.empty(rows, cols, dtype=dtype, device=dev) if out is None else out
        _ck(_lib.anakin_ckpt_unpack(DTYPES[dtype], rows, cols, _ptr(ck.codes), _ptr(ck.scales), _ptr(out), _ld(out), stream))
    return out


def ckpt_backward(ck: Checkpoint, dy: torch.Tensor, act: str = "relu", out: torch.Tensor | None = None) -> torch.Tensor:
    """dy * act'(x) with x from its checkpoint (anakin_ckpt_backward); `out` may be dy itself."""
    dev, rows, cols = _checkpoint(ck)
    _, _, ld = _matrix("dy", dy, dev, dy.dtype if isinstance(dy, torch.Tensor) else None, (rows, cols))
    a = _one_of(ACTS, "act", act)
    with _Device(dev) as stream:
        out = _like("out", out, dy)
        _ck(_lib.anakin_ckpt_backward(DTYPES[dy.dtype], a, rows, cols, _ptr(ck.codes), _ptr(ck.scales), _ptr(dy), ld, _ptr(out), _ld(out), stream))
    return out


def ckpt_weight_grad(ck: Checkpoint, dy: torch.Tensor, act: str = "identity", out: torch.Tensor | None = None, accumulate: bool = False,
                     status: torch.Tensor | None = None) -> torch.Tensor:
    """act(x)^T dy, f32 [cols][n], with x from its checkpoint (anakin_ckpt_weight_grad); accumulate adds to `out`.  `status` (int32 [1], zeroed by
    the caller) takes the device status bits."""
    dev, rows, cols = _checkpoint(ck)
    r, n, ld = _matrix("dy", dy, dev, dy.dtype if isinstance(dy, torch.Tensor) else None, (rows, dy.shape[1]) if isinstance(dy, torch.Tensor) and dy.dim() == 2 else (rows, 1))
    a = _one_of(ACTS, "act", act)
    if a > 1:
        _refuse("act is identity or relu here: checkpoint the activation's output", E_UNSUPPORTED_CFG)
    if accumulate and out is None:
        _refuse("accumulate adds to `out`")
    _on(dev, "status", status, torch.int32, (1,))
    with _Device(dev) as stream:
        if out is None:
            out = torch.empty(cols, n, device=dev)
        else:
            _matrix("out", out, dev, torch.float32, (cols, n))
        size = C.c_size_t(0)
        _ck(_lib.anakin_ckpt_weight_grad_workspace_bytes(DTYPES[dy.dtype], rows, cols, n, C.byref(size)))
        ws = torch.empty(size.value, dtype=torch.uint8, device=dev)
        _ck(_lib.anakin_ckpt_weight_grad(DTYPES[dy.dtype], a, rows, cols, n, _ptr(ck.codes), _ptr(ck.scales), _ptr(dy), ld, _ptr(out), _ld(out),
                                         int(accumulate), _ptr(ws), ws.numel(), _ptr(status), stream))
    return out
