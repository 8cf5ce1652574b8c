"""Policies over token vocabularies, and activation checkpoints in 8 bits: Python functions over the stateless calls of include/anakin.h
(anakin_token_*, anakin_ckpt_*), which say what each computes.

Argument marshalling only.  Tensors lie on one CUDA device; work is enqueued on that device's current torch stream, outputs and
workspaces come from torch's allocator on that stream, nothing synchronises, and every call may be captured into a CUDA graph.  Gradients
are outputs (`logits.backward(dlogits)` hands one to autograd); the inputs are not differentiated through.  What a call refuses it
refuses with AnakinError before anything is enqueued.
"""
from __future__ import annotations

import ctypes as C
import functools
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
_lib.anakin_ckpt_weight_grad_workspace_bytes.argtypes = [C.c_int, _i64, _i64, _i64, C.c_int, _sz]
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


# The smallest of these calls cost the host more than the GPU, so the checks below are few attribute look-ups each.
_F32, _U8, _Tensor, _empty = torch.float32, torch.uint8, torch.Tensor, torch.empty
_TOKEN_ROWS = C.sizeof(TokenRows)
_stream_of = torch._C._cuda_getCurrentRawStream  # a device's current stream as an integer
_INTS, _FLAGS = (torch.int64, torch.int32), (torch.bool, torch.uint8)


def _vector(name: str, t, n: int, dev: torch.device, dtypes=(_F32,)) -> int | None:
    """Address of t, a dense vector of n numbers on that device; None stays None."""
    if t is None:
        return None
    if not isinstance(t, _Tensor) or t.dtype not in dtypes or t.shape != (n,) or t.device != dev or not t.is_contiguous():
        _refuse(f"{name}: a dense vector of {n} numbers ({', '.join(map(str, dtypes))}) on {dev} is needed")
    return t.data_ptr()


def _matrix(name: str, t, dev=None, dtype=None, shape=None) -> tuple[int, int, int]:
    """(rows, cols, elements from row to row) of a matrix whose rows are dense."""
    if not isinstance(t, _Tensor) or not t.is_cuda or t.dtype not in DTYPES or t.dim() != 2:
        _refuse(f"{name}: a CUDA matrix of float32, bfloat16 or float16 is needed")
    (rows, cols), (ld, step) = t.shape, t.stride()
    if cols < 1 or (dev is not None and t.device != dev) or (dtype is not None and t.dtype is not dtype) or (shape is not None and (rows, cols) != shape):
        _refuse(f"{name}: {dtype or 'a matrix'} of shape {shape or '(rows, one column at least)'} on {dev or 'a GPU'} is needed")
    if rows <= 1:
        ld = cols
    if (cols > 1 and step != 1) or ld < cols:
        _refuse(f"{name}: columns have to lie side by side, and rows one after the other")
    return rows, cols, ld


_gpus = functools.lru_cache(maxsize=None)(torch.cuda.device_count)


def _on_its_device(call):
    """The call with its tensors' GPU as the current one."""

    @functools.wraps(call)
    def wrapped(*args, **kw):
        if _gpus() > 1:
            for a in (*args, *kw.values()):
                a = a.codes if isinstance(a, Checkpoint) else a
                if isinstance(a, _Tensor) and a.is_cuda:
                    with torch.cuda.device(a.device):
                        return call(*args, **kw)
        return call(*args, **kw)

    return wrapped


def _token_rows(dev, n, tokens, mask, offsets, logits=None, vocab=0, ld=0, scale=1.0) -> TokenRows:
    r = TokenRows(_TOKEN_ROWS, 0, n, vocab, ld)
    r.scale = scale
    if logits is not None:
        r.dtype, r.logits = DTYPES[logits.dtype], logits.data_ptr()
    if tokens is not None:
        r.tokens, r.token_bytes = _vector("tokens", tokens, n, dev, _INTS), tokens.element_size()
    if mask is not None:
        r.mask = _vector("mask", mask, n, dev, _FLAGS)
    if offsets is not None:
        count = offsets.numel() if isinstance(offsets, _Tensor) else 0
        if count < 1:
            _refuse("offsets: one number more than there are sequences")
        r.offsets, r.offset_bytes, r.sequences = _vector("offsets", offsets, count, dev, _INTS), offsets.element_size(), count - 1
    return r


@functools.lru_cache(maxsize=256)
def _workspace_bytes(rows: int, sequences: int) -> int:
    n = C.c_size_t(0)
    _ck(_lib.anakin_token_workspace_bytes(rows, sequences, C.byref(n)))
    return n.value


def _like(name: str, out, like: torch.Tensor) -> tuple[torch.Tensor, int]:
    """A matrix like `like`, and its elements from row to row."""
    if out is None:
        if like.is_contiguous():
            return torch.empty_like(like), like.shape[1]
        return _empty(like.shape, dtype=like.dtype, device=like.device), like.shape[1]
    return out, _matrix(name, out, like.device, like.dtype, tuple(like.shape))[2]


@_on_its_device
def logp(logits: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, mask: torch.Tensor | None = None, entropy: bool = True) -> TokenLogp:
    """Log-probability of every row's token under softmax(scale * logits), and the entropy (anakin_token_logp)."""
    n, vocab, ld = _matrix("logits", logits)
    dev = logits.device
    if tokens is None:
        _refuse("tokens are needed")
    stream = _stream_of(dev.index)
    rows = _token_rows(dev, n, tokens, mask, None, logits, vocab, ld, scale)
    norm, lp, ent = _empty(n, 2, device=dev), _empty(n, device=dev), _empty(n, device=dev) if entropy else None
    _ck(_lib.anakin_token_logp(rows, lp.data_ptr(), ent.data_ptr() if entropy else None, norm.data_ptr(), stream))
    return TokenLogp(lp, ent, norm)


@_on_its_device
def logp_backward(logits: torch.Tensor, tokens: torch.Tensor, norm: torch.Tensor, dlogp: torch.Tensor, entropy: torch.Tensor | None = None,
                  dentropy: torch.Tensor | None = None, scale: float = 1.0, mask: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """Gradient of the logits from those of logp and entropy (anakin_token_logp_backward).  norm and entropy come from logp() with the same
    tokens, scale and mask; `out` may be the logits themselves."""
    n, vocab, ld = _matrix("logits", logits)
    dev = logits.device
    if tokens is None or dlogp is None or (dentropy is not None and entropy is None):
        _refuse("tokens, norm and dlogp are needed, and entropy with dentropy")
    if _matrix("norm", norm, dev, _F32, (n, 2))[2] != 2:
        _refuse("norm: its rows lie one behind the other")
    stream = _stream_of(dev.index)
    rows = _token_rows(dev, n, tokens, mask, None, logits, vocab, ld, scale)
    out, ld_out = _like("out", out, logits)
    _ck(_lib.anakin_token_logp_backward(rows, norm.data_ptr(), _vector("entropy", entropy, n, dev), _vector("dlogp", dlogp, n, dev),
                                        _vector("dentropy", dentropy, n, dev), out.data_ptr(), ld_out, stream))
    return out


@_on_its_device
def policy_loss(objective: PolicyObjective, logp: torch.Tensor, old_logp: torch.Tensor | None, adv: torch.Tensor, ref_logp: torch.Tensor | None = None,
                entropy: torch.Tensor | None = None, mask: torch.Tensor | None = None, offsets: torch.Tensor | None = None,
                tokens: torch.Tensor | None = None) -> PolicyLoss:
    """The clipped policy loss from log-probabilities, and its gradients (anakin_token_policy_loss)."""
    if not isinstance(logp, torch.Tensor) or not logp.is_cuda or logp.dim() != 1:
        _refuse("logp: a CUDA vector is needed")
    if adv is None or (objective.kl != 0 and ref_logp is None):
        _refuse("adv is needed, and ref_logp with a KL term")
    n, dev = logp.shape[0], logp.device
    stream = _stream_of(dev.index)
    rows = _token_rows(dev, n, tokens, mask, offsets)
    size = _workspace_bytes(n, rows.sequences)
    ws = _empty(size, dtype=_U8, device=dev)
    stats, dlogp, dentropy = _empty(len(POLICY_STATS), device=dev), _empty(n, device=dev), _empty(n, device=dev) if entropy is not None else None
    _ck(_lib.anakin_token_policy_loss(rows, objective, _vector("logp", logp, n, dev), _vector("old_logp", old_logp, n, dev), _vector("adv", adv, n, dev),
                                      _vector("ref_logp", ref_logp, n, dev), _vector("entropy", entropy, n, dev), stats.data_ptr(), dlogp.data_ptr(),
                                      None if dentropy is None else dentropy.data_ptr(), ws.data_ptr(), size, stream))
    return PolicyLoss(stats, dlogp, dentropy)


@_on_its_device
def policy_grad(objective: PolicyObjective, logits: torch.Tensor, tokens: torch.Tensor, old_logp: torch.Tensor | None, adv: torch.Tensor,
                ref_logp: torch.Tensor | None = None, mask: torch.Tensor | None = None, offsets: torch.Tensor | None = None, scale: float = 1.0,
                out: torch.Tensor | None = None) -> PolicyGrad:
    """The clipped policy loss from logits, with the gradient of the logits (anakin_token_policy_grad); `out` may be the logits themselves."""
    n, vocab, ld = _matrix("logits", logits)
    dev = logits.device
    if tokens is None or adv is None or (objective.kl != 0 and ref_logp is None):
        _refuse("tokens and adv are needed, and ref_logp with a KL term")
    stream = _stream_of(dev.index)
    rows = _token_rows(dev, n, tokens, mask, offsets, logits, vocab, ld, scale)
    size = _workspace_bytes(n, rows.sequences)
    ws = _empty(size, dtype=_U8, device=dev)
    stats, lp, ent = _empty(len(POLICY_STATS), device=dev), _empty(n, device=dev), _empty(n, device=dev)
    out, ld_out = _like("out", out, logits)
    _ck(_lib.anakin_token_policy_grad(rows, objective, _vector("old_logp", old_logp, n, dev), _vector("adv", adv, n, dev),
                                      _vector("ref_logp", ref_logp, n, dev), stats.data_ptr(), lp.data_ptr(), ent.data_ptr(), out.data_ptr(), ld_out,
                                      ws.data_ptr(), size, stream))
    return PolicyGrad(stats, lp, ent, out)


@_on_its_device
def preference_loss(objective: PreferenceObjective, logp: torch.Tensor, offsets: torch.Tensor, ref_logp: torch.Tensor | None = None,
                    mask: torch.Tensor | None = None, tokens: torch.Tensor | None = None) -> PreferenceLoss:
    """The preference loss over pairs of sequences, the preferred ones first, and its gradient (anakin_token_preference_loss)."""
    if not isinstance(logp, torch.Tensor) or not logp.is_cuda or logp.dim() != 1:
        _refuse("logp: a CUDA vector is needed")
    if not isinstance(offsets, torch.Tensor) or offsets.numel() % 2 == 0:
        _refuse("offsets of an even number of sequences are needed")
    n, dev = logp.shape[0], logp.device
    stream = _stream_of(dev.index)
    rows = _token_rows(dev, n, tokens, mask, offsets)
    size = _workspace_bytes(n, rows.sequences)
    ws = _empty(size, dtype=_U8, device=dev)
    stats, margin, dlogp = _empty(len(PREFERENCE_STATS), device=dev), _empty(rows.sequences // 2, device=dev), _empty(n, device=dev)
    _ck(_lib.anakin_token_preference_loss(rows, objective, _vector("logp", logp, n, dev), _vector("ref_logp", ref_logp, n, dev), stats.data_ptr(),
                                          margin.data_ptr(), dlogp.data_ptr(), ws.data_ptr(), size, stream))
    return PreferenceLoss(stats, margin, dlogp)


def _checkpoint(ck: Checkpoint) -> tuple[torch.device, int, int]:
    codes, scales, cols = ck
    blocks = (cols + 31) // 32
    if not isinstance(codes, _Tensor) or codes.dtype is not _U8 or not codes.is_cuda or codes.dim() != 2 or cols < 1 or codes.shape[1] != blocks * 32 or not codes.is_contiguous():
        _refuse(f"codes: a dense CUDA matrix of uint8 with {blocks * 32} columns is needed")
    rows, dev = codes.shape[0], codes.device
    if not isinstance(scales, _Tensor) or scales.dtype is not _U8 or scales.shape != (rows, blocks) or scales.device != dev or not scales.is_contiguous():
        _refuse(f"scales: a dense matrix of uint8, {rows} x {blocks}, is needed beside the codes")
    return dev, rows, cols


@_on_its_device
def ckpt_forward(x: torch.Tensor, act: str = "relu", y: bool = True, out: torch.Tensor | None = None) -> tuple[torch.Tensor | None, Checkpoint]:
    """act(x) (None with y=False) and the checkpoint of x in 8 bits (anakin_ckpt_forward); `out` may be x itself."""
    rows, cols, ld = _matrix("x", x)
    a, dev, blocks = _one_of(ACTS, "act", act), x.device, (cols + 31) // 32
    stream = _stream_of(dev.index)
    res, ldy = _like("out", out, x) if y else (None, 0)
    codes = _empty(rows, blocks * 32, dtype=_U8, device=dev)
    scales = _empty(rows, blocks, dtype=_U8, device=dev)
    _ck(_lib.anakin_ckpt_forward(DTYPES[x.dtype], a, rows, cols, x.data_ptr(), ld, res.data_ptr() if y else None, ldy, codes.data_ptr(), scales.data_ptr(), stream))
    return res, Checkpoint(codes, scales, cols)


@_on_its_device
def ckpt_unpack(ck: Checkpoint, dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None) -> torch.Tensor:
    """The values that a checkpoint holds (anakin_ckpt_unpack)."""
    dev, rows, cols = _checkpoint(ck)
    if out is not None:
        ld, dtype = _matrix("out", out, dev, None, (rows, cols))[2], out.dtype
    elif dtype not in DTYPES:
        _refuse("float32, bfloat16 or float16")
    stream = _stream_of(dev.index)
    if out is None:
        out, ld = _empty(rows, cols, dtype=dtype, device=dev), cols
    _ck(_lib.anakin_ckpt_unpack(DTYPES[dtype], rows, cols, ck.codes.data_ptr(), ck.scales.data_ptr(), out.data_ptr(), ld, stream))
    return out


@_on_its_device
def ckpt_backward(ck: Checkpoint, dy: torch.Tensor, act: str = "relu", out: torch.Tensor | None = None) -> torch.Tensor:
    """dy * act'(x) with x from its checkpoint (anakin_ckpt_backward); `out` may be dy itself."""
    dev, rows, cols = _checkpoint(ck)
    ld, a = _matrix("dy", dy, dev, None, (rows, cols))[2], _one_of(ACTS, "act", act)
    stream = _stream_of(dev.index)
    out, ldx = _like("out", out, dy)
    _ck(_lib.anakin_ckpt_backward(DTYPES[dy.dtype], a, rows, cols, ck.codes.data_ptr(), ck.scales.data_ptr(), dy.data_ptr(), ld, out.data_ptr(), ldx, stream))
    return out


@functools.lru_cache(maxsize=256)
def _weight_grad_bytes(dtype: int, rows: int, cols: int, n: int, aligned: bool) -> int:
    size = C.c_size_t(0)
    _ck(_lib.anakin_ckpt_weight_grad_workspace_bytes(dtype, rows, cols, n, int(aligned), C.byref(size)))
    return size.value


@_on_its_device
def ckpt_weight_grad(ck: Checkpoint, dy: torch.Tensor, act: str = "identity", out: torch.Tensor | None = None, accumulate: bool = False,
                     status: torch.Tensor | None = None) -> torch.Tensor:
    """act(x)^T dy, f32 [cols][n], with x from its checkpoint (anakin_ckpt_weight_grad); accumulate adds to `out`.  `status` (int32 [1], zeroed by
    the caller) takes the device status bits."""
    dev, rows, cols = _checkpoint(ck)
    r, n, ld = _matrix("dy", dy, dev)
    a, dt = _one_of(ACTS, "act", act), DTYPES[dy.dtype]
    if r != rows:
        _refuse(f"dy: {rows} rows are needed")
    if a > 1:
        _refuse("act is identity or relu here: checkpoint the activation's output", E_UNSUPPORTED_CFG)
    if out is not None:
        ldw = _matrix("out", out, dev, _F32, (cols, n))[2]
    elif accumulate:
        _refuse("accumulate adds to `out`")
    stream = _stream_of(dev.index)
    if out is None:
        out, ldw = _empty(cols, n, device=dev), n
    at = dy.data_ptr()
    size = _weight_grad_bytes(dt, rows, cols, n, (at | ld * dy.element_size()) % 16 == 0)
    ws = _empty(size, dtype=_U8, device=dev)
    _ck(_lib.anakin_ckpt_weight_grad(dt, a, rows, cols, n, ck.codes.data_ptr(), ck.scales.data_ptr(), at, ld, out.data_ptr(), ldw,
                                     int(accumulate), ws.data_ptr(), size, _vector("status", status, 1, dev, (torch.int32,)), stream))
    return out
