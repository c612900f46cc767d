"""Cross entropy of tokens over a vocabulary, from hidden states and an output matrix, without keeping the logits, and its
gradients.

Thin binding over the ``stq_vocab_*`` calls of libstq, in the manner of ``q8``: torch supplies memory and streams, matrices have
unit stride along a row and any pitch, each call enqueues its work on the current stream of the handle's device (or on
``stream``) and does not synchronise, except where it needs more workspace than any call before it.  One handle serves one
stream at a time.

Tokens whose target is ``ignore_index`` have loss 0, lse 0 and no gradient; nothing is computed of them.  Any other target
outside the vocabulary cannot be refused without waiting for the device: it gives NaN.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional

import torch

from . import stq
from .q8 import _BF16, _F32, _empty, _mat, _On, _out_dtype, _raw_stream, _vec

MAX_TOKENS, MAX_WIDTH = 262144, 65536      # STQ_VOCAB_MAX_*

_fn = None


def _lib() -> C.CDLL:
    global _fn
    if _fn is None:
        L = stq.lib()
        vp, u64, i64, u32, i = C.c_void_p, C.c_uint64, C.c_int64, C.c_uint32, C.c_int
        L.stq_vocab_loss.argtypes = [vp, vp, u64, vp, u64, vp, vp, i64, u64, u32, u32, vp, vp, vp]
        L.stq_vocab_loss_backward.argtypes = [vp, vp, vp, u64, vp, u64, vp, vp, i64, vp, u64, u32, u32, vp, u64, vp, u64, i, vp, vp]
        _fn = L
    return _fn


class LossOut(NamedTuple):
    loss: torch.Tensor               # float32 [t]
    lse: torch.Tensor                # float32 [t]: log of the sum of exp of a token's logits


class LossGrads(NamedTuple):
    dx: Optional[torch.Tensor]       # bfloat16 [t, d]
    dw: Optional[torch.Tensor]       # [v, d]
    dbias: Optional[torch.Tensor]    # float32 [v]


def _targets(target: torch.Tensor, dev: int, t: int):
    if target.shape != (t,) or target.dtype is not torch.int64 or not target.is_contiguous():
        raise ValueError(f"target is a contiguous int64 vector of {t}")
    if target.get_device() != dev:
        raise ValueError("target lives on the handle's device")


def _given(dev, x, w, target, bias):
    ldx = _mat("x", x, dev, _BF16)
    t, d = x.shape
    ldw = _mat("w", w, dev, _BF16, None, d)
    v = w.shape[0]
    _targets(target, dev, t)
    if bias is not None:
        _vec("bias", bias, dev, v)
    if t > MAX_TOKENS or d > MAX_WIDTH:
        raise ValueError(f"at most {MAX_TOKENS} tokens of {MAX_WIDTH} columns")
    return t, d, v, ldx, ldw


def loss(handle: stq.Handle, x: torch.Tensor, w: torch.Tensor, target: torch.Tensor, *, bias: torch.Tensor | None = None,
         ignore_index: int = -100, stream=None) -> LossOut:
    """Cross entropy of ``target`` (int64 [t]) under the logits x [t, d] times w [v, d] transposed (both bfloat16), plus bias
    (float32 [v])."""
    if stream is not None:
        with _On(stream, (x, w, target, bias)):
            return loss(handle, x, w, target, bias=bias, ignore_index=ignore_index)
    dev = handle.device
    t, d, v, ldx, ldw = _given(dev, x, w, target, bias)
    device = x.device
    out = _empty((t,), (1,), dtype=_F32, device=device)
    lse = _empty((t,), (1,), dtype=_F32, device=device)
    rc = (_fn or _lib()).stq_vocab_loss(handle._h, x.data_ptr(), ldx, w.data_ptr(), ldw, None if bias is None else bias.data_ptr(),
                                        target.data_ptr(), ignore_index, t, v, d, out.data_ptr(), lse.data_ptr(), _raw_stream(dev))
    if rc:
        handle._check(rc, "stq_vocab_loss")
    return LossOut(out, lse)


def loss_backward(handle: stq.Handle, dloss: torch.Tensor, x: torch.Tensor, w: torch.Tensor, target: torch.Tensor, lse: torch.Tensor, *,
                  bias: torch.Tensor | None = None, ignore_index: int = -100, dtype=torch.bfloat16, want_dx: bool = True,
                  want_dw: bool = True, want_dbias: bool | None = None, stream=None) -> LossGrads:
    """Gradients of ``loss`` for ``dloss`` (float32 [t]).  ``dtype`` is that of dw: with bfloat16 the logits' gradients are
    rounded to bfloat16 on the way, with float32 they are not, for dw (at three times the cost of its product).  ``want_*``: what
    is formed (dbias by default if there is a bias)."""
    if stream is not None:
        with _On(stream, (dloss, x, w, target, lse, bias)):
            return loss_backward(handle, dloss, x, w, target, lse, bias=bias, ignore_index=ignore_index, dtype=dtype, want_dx=want_dx,
                                 want_dw=want_dw, want_dbias=want_dbias)
    dev = handle.device
    odt = _out_dtype(dtype)
    t, d, v, ldx, ldw = _given(dev, x, w, target, bias)
    _vec("dloss", dloss, dev, t)
    _vec("lse", lse, dev, t)
    device = x.device
    dx = _empty((t, d), (d, 1), dtype=_BF16, device=device) if want_dx else None
    dw = _empty((v, d), (d, 1), dtype=dtype, device=device) if want_dw else None
    if want_dbias is None:
        want_dbias = bias is not None
    db = _empty((v,), (1,), dtype=_F32, device=device) if want_dbias else None
    rc = (_fn or _lib()).stq_vocab_loss_backward(
        handle._h, dloss.data_ptr(), x.data_ptr(), ldx, w.data_ptr(), ldw, None if bias is None else bias.data_ptr(), target.data_ptr(),
        ignore_index, lse.data_ptr(), t, v, d, None if dx is None else dx.data_ptr(), d, None if dw is None else dw.data_ptr(), d, odt,
        None if db is None else db.data_ptr(), _raw_stream(dev))
    if rc:
        handle._check(rc, "stq_vocab_loss_backward")
    return LossGrads(dx, dw, db)
