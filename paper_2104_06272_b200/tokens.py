"""Policies over token vocabularies, and activation checkpoints in 8 bits: Python functions over the stateless calls of include/anakin.h
(anakin_token_*, anakin_ckpt_*), which say what each computes.

Argument marshalling only, done in C++ (csrc/tokens_host.cpp), as the smallest calls cost the host more than the GPU.  Tensors lie on one
CUDA device; work is enqueued on that device's current torch stream, outputs and workspaces come from torch's allocator on that stream,
nothing synchronises, and every call may be captured into a CUDA graph.  Gradients are outputs (`logits.backward(dlogits)` hands one to
autograd); the inputs are not differentiated through.  What a call refuses it refuses with AnakinError before anything is enqueued.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple

import torch

from .binding import E_INVALID_ARG, AnakinError, lib

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


try:
    from . import _tokens_host as _host
except ImportError as e:
    raise ImportError(f"{e}; build it with `python -m paper_2104_06272_b200.build`") from e
_host.set_error(AnakinError)
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


def _refuse(why: str):
    raise AnakinError(E_INVALID_ARG, why)


def _one_of(table: dict, name: str, key: str) -> int:
    if key not in table:
        _refuse(f"{name} is one of {', '.join(table)}")
    return table[key]


def logp(logits: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, mask: torch.Tensor | None = None, entropy: bool = True) -> TokenLogp:
    """Log-probability of every row's token under softmax(scale * logits), and the entropy (anakin_token_logp).  No grad_fn, whatever the logits have:
    logp_backward is the gradient."""
    return TokenLogp._make(_host.logp(logits, tokens, scale, mask, entropy))


def logp_backward(logits: torch.Tensor, tokens: torch.Tensor, norm: torch.Tensor, dlogp: torch.Tensor, entropy: torch.Tensor | None = None,
                  dentropy: torch.Tensor | None = None, scale: float = 1.0, mask: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """Gradient of the logits from those of logp and entropy (anakin_token_logp_backward).  norm and entropy come from logp() with the same
    tokens, scale and mask; `out` may be the logits themselves."""
    return _host.logp_backward(logits, tokens, norm, dlogp, entropy, dentropy, scale, mask, out)


def policy_loss(objective: PolicyObjective, logp: torch.Tensor, old_logp: torch.Tensor | None, adv: torch.Tensor, ref_logp: torch.Tensor | None = None,
                entropy: torch.Tensor | None = None, mask: torch.Tensor | None = None, offsets: torch.Tensor | None = None,
                tokens: torch.Tensor | None = None) -> PolicyLoss:
    """The clipped policy loss from log-probabilities, and its gradients (anakin_token_policy_loss)."""
    return PolicyLoss._make(_host.policy_loss(objective, logp, old_logp, adv, ref_logp, entropy, mask, offsets, tokens))


def policy_grad(objective: PolicyObjective, logits: torch.Tensor, tokens: torch.Tensor, old_logp: torch.Tensor | None, adv: torch.Tensor,
                ref_logp: torch.Tensor | None = None, mask: torch.Tensor | None = None, offsets: torch.Tensor | None = None, scale: float = 1.0,
                out: torch.Tensor | None = None) -> PolicyGrad:
    """The clipped policy loss from logits, with the gradient of the logits (anakin_token_policy_grad); `out` may be the logits themselves."""
    return PolicyGrad._make(_host.policy_grad(objective, logits, tokens, old_logp, adv, ref_logp, mask, offsets, scale, out))


def preference_loss(objective: PreferenceObjective, logp: torch.Tensor, offsets: torch.Tensor, ref_logp: torch.Tensor | None = None,
                    mask: torch.Tensor | None = None, tokens: torch.Tensor | None = None) -> PreferenceLoss:
    """The preference loss over pairs of sequences, the preferred ones first, and its gradient (anakin_token_preference_loss)."""
    return PreferenceLoss._make(_host.preference_loss(objective, logp, offsets, ref_logp, mask, tokens))


def ckpt_forward(x: torch.Tensor, act: str = "relu", y: bool = True, out: torch.Tensor | None = None) -> tuple[torch.Tensor | None, Checkpoint]:
    """act(x) (None with y=False) and the checkpoint of x in 8 bits (anakin_ckpt_forward); `out` may be x itself.  The result has no grad_fn, whatever x has: in a
    network under autograd the gradient would end here.  Its backward pass is ckpt_backward."""
    res, codes, scales = _host.ckpt_forward(x, _one_of(ACTS, "act", act), y, out)
    return res, Checkpoint(codes, scales, x.shape[1])


def ckpt_unpack(ck: Checkpoint, dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None) -> torch.Tensor:
    """The values that a checkpoint holds (anakin_ckpt_unpack)."""
    if out is None and dtype not in DTYPES:
        _refuse("float32, bfloat16 or float16")
    return _host.ckpt_unpack(*ck, DTYPES.get(dtype, 0), out)


def ckpt_backward(ck: Checkpoint, dy: torch.Tensor, act: str = "relu", out: torch.Tensor | None = None) -> torch.Tensor:
    """dy * act'(x) with x from its checkpoint (anakin_ckpt_backward); `out` may be dy itself."""
    return _host.ckpt_backward(*ck, dy, _one_of(ACTS, "act", act), out)


def ckpt_weight_grad(ck: Checkpoint, dy: torch.Tensor, act: str = "identity", out: torch.Tensor | None = None, accumulate: bool = False,
                     status: torch.Tensor | None = None) -> torch.Tensor:
    """act(x)^T dy, f32 [cols][n], with x from its checkpoint (anakin_ckpt_weight_grad); accumulate adds to `out`.  `status` (int32 [1], zeroed by
    the caller) takes the device status bits."""
    return _host.ckpt_weight_grad(*ck, dy, _one_of(ACTS, "act", act), out, accumulate, status)
