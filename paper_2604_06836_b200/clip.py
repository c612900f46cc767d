"""The 2-norm of all gradients together, the factor that clips them, and the clipped gradients.

Thin binding over ``stq_grad_norm`` and ``stq_grad_clip``, in the manner of ``q8``: everything stays on the device and is enqueued on
the current stream of the handle's device (or on ``stream``).  ``optim.STQAdamW(max_norm=...)`` takes the factor into its step, which
then clips without writing the gradients; ``clip_grads`` is for every other optimizer.

Gradients are float32, bfloat16 or float16, each its own, in any dense layout (no gaps, no overlap); None is passed over.  A
generator of them will do.

Where each rank of a job has a part of the parameters (``multi.partition``), this is the norm of one rank's part: the squares of the norms
have to be added over the ranks before a factor is taken from them.
"""
from __future__ import annotations

import ctypes as C
import importlib
import math
from typing import NamedTuple, Optional, Sequence

import torch

from . import stq
from .build import lists_name
from .q8 import _F32, _empty, _On, _raw_stream

_fn = _lists = None


def _lib() -> C.CDLL:
    global _fn, _lists
    if _fn is None:
        L = stq.lib()
        name = lists_name(torch.__version__)
        try:
            _lists = importlib.import_module("." + name, __package__)
        except ModuleNotFoundError:
            raise RuntimeError(f"{name} is missing (built for another torch or Python?): build it with `python -m paper_2604_06836_b200.build`") from None
        vp, i, f = C.c_void_p, C.c_int, C.c_float
        for fn in (L.stq_grad_norm, L.stq_grad_clip):
            fn.argtypes = [vp, C.c_char_p, i, vp, f, f, vp, vp, vp, vp]
        _fn = L
    return _fn


class Norm(NamedTuple):
    norm: torch.Tensor       # float32, no dimensions: the norm, unscaled
    factor: torch.Tensor     # float32, no dimensions: what a gradient is multiplied with


def _scalar(name, t, dev):
    if t is None:
        return None
    if t.numel() != 1 or t.dtype is not _F32 or t.get_device() != dev:
        raise ValueError(f"{name} is one float32 on the handle's device")
    return t.data_ptr()


def _kept(tensors):
    """A list of them that can be gone through more than once (a generator cannot)."""
    return tensors if tensors is None or isinstance(tensors, (list, tuple)) else list(tensors)


def _call(clipped: bool, handle, grads, out, max_norm, inv_scale, found_inf, eps) -> Norm:
    L, dev = _fn or _lib(), handle.device
    max_norm = math.inf if max_norm is None else float(max_norm)
    if not max_norm > 0.0 or not 0.0 <= eps < math.inf:
        raise ValueError("max_norm is positive (None: no clipping), eps is not negative")
    inv, flag = _scalar("inv_scale", inv_scale, dev), _scalar("found_inf", found_inf, dev)
    rows, n = _lists.rows(grads, out, dev)
    both = _empty((2,), (1,), dtype=_F32, device=f"cuda:{dev}")
    at = both.data_ptr()
    fn = L.stq_grad_clip if clipped else L.stq_grad_norm
    rc = fn(handle._h, rows, n, inv, max_norm, eps, at, at + 4, flag, _raw_stream(dev))
    if rc:
        handle._check(rc, fn.__name__)
    if clipped:
        _lists.written(grads if out is None else out)
    return Norm(*both.unbind())


def grad_norm(handle: stq.Handle, grads: Sequence[Optional[torch.Tensor]], *, max_norm: float | None = None,
              inv_scale: torch.Tensor | None = None, found_inf: torch.Tensor | None = None, eps: float = 1e-6, stream=None) -> Norm:
    """norm = inv_scale * 2-norm of all gradients, factor = inv_scale * min(1, max_norm / (norm + eps)).  ``inv_scale``: one float32
    on the device (1 / loss scale); ``found_inf``: one float32 on the device, set to 1 where the norm is not finite."""
    grads = _kept(grads)
    if stream is not None:
        with _On(stream, (*grads, inv_scale, found_inf)):
            return grad_norm(handle, grads, max_norm=max_norm, inv_scale=inv_scale, found_inf=found_inf, eps=eps)
    return _call(False, handle, grads, None, max_norm, inv_scale, found_inf, eps)


def clip_grads(handle: stq.Handle, grads: Sequence[Optional[torch.Tensor]], max_norm: float | None, *,
               inv_scale: torch.Tensor | None = None, found_inf: torch.Tensor | None = None, eps: float = 1e-6,
               out: Sequence[Optional[torch.Tensor]] | None = None, stream=None) -> Norm:
    """``grad_norm``, and the gradients times the factor: in place, or written to ``out`` (a tensor for each gradient, of its type or
    float32; the gradients stay as they are)."""
    grads, out = _kept(grads), _kept(out)
    if stream is not None:
        with _On(stream, (*grads, *(out or ()), inv_scale, found_inf)):
            return clip_grads(handle, grads, max_norm, inv_scale=inv_scale, found_inf=found_inf, eps=eps, out=out)
    return _call(True, handle, grads, out, max_norm, inv_scale, found_inf, eps)
