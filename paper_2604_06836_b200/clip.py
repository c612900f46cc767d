"""The 2-norm of all gradients together, the factor that clips them, and the clipped gradients.

Thin binding over ``stq_grad_norm`` and ``stq_grad_clip``, in the manner of ``q8``: everything stays on the device and is enqueued on
the current stream of the handle's device (or on ``stream``).  ``optim.STQAdamW(max_norm=...)`` takes the factor into its step, which
then clips without writing the gradients; ``clip_grads`` is for every other optimizer.

Gradients are float32, bfloat16 or float16, each its own, in any dense layout (no gaps, no overlap); None is passed over.
"""
from __future__ import annotations

import ctypes as C
import math
from array import array
from typing import NamedTuple, Optional, Sequence

import torch

from . import stq
from .q8 import _F32, _empty, _On, _raw_stream

_address_of, _length_of, _device_of = torch.Tensor.data_ptr, torch.Tensor.numel, torch.Tensor.get_device
_DT = {torch.float32: stq.GRAD_F32, torch.bfloat16: stq.GRAD_BF16, torch.float16: stq.GRAD_F16}

_fn = None


def _lib() -> C.CDLL:
    global _fn
    if _fn is None:
        L = stq.lib()
        vp, i, f = C.c_void_p, C.c_int, C.c_float
        for fn in (L.stq_grad_norm, L.stq_grad_clip):
            fn.argtypes = [vp, vp, i, vp, f, f, vp, vp, vp, vp]
        _fn = L
    return _fn


class Norm(NamedTuple):
    norm: torch.Tensor       # float32, no dimensions: the norm, unscaled
    factor: torch.Tensor     # float32, no dimensions: what a gradient is multiplied with


def _dense(t: torch.Tensor) -> bool:
    """Whether the elements fill a range of memory, in some order."""
    if t.is_contiguous():
        return True
    expect = 1
    for size, stride in sorted(((s, d) for s, d in zip(t.shape, t.stride()) if s != 1), key=lambda x: x[1]):
        if stride != expect:
            return False
        expect *= size
    return True


def _refuse(name, t, dev):
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} are tensors")
    if t.get_device() != dev:
        raise ValueError(f"{name} live on the handle's device")
    if t.dtype not in _DT:
        raise ValueError(f"{name} are float32, bfloat16 or float16, not {t.dtype}")
    raise ValueError(f"{name} are dense: no gaps, no overlap")


def _table(grads, out, dev):
    """Rows of the call as one array of integers (the layout of stq_grad), and their number.  (A model has hundreds of tensors: one
    pass of the interpreter for each thing to know of them, and what is wrong is found out only once something is.)"""
    if any(g is None for g in grads):
        out = None if out is None else [o for g, o in zip(grads, out) if g is not None]
        grads = [g for g in grads if g is not None]
    n = len(grads)
    try:
        types = [_DT[g.dtype] for g in grads]
        if any(d != dev for d in map(_device_of, grads)) or not all(g.is_contiguous() or _dense(g) for g in grads):
            raise KeyError
    except (KeyError, AttributeError):
        for g in grads:
            if not isinstance(g, torch.Tensor) or g.dtype not in _DT or g.get_device() != dev or not _dense(g):
                _refuse("gradients", g, dev)
        raise
    rows = array("Q", bytes(32 * n))
    rows[0::4] = rows[1::4] = array("Q", map(_address_of, grads))
    rows[2::4] = array("Q", map(_length_of, grads))
    if out is not None:
        for g, o, dt in zip(grads, out, types):
            if not isinstance(o, torch.Tensor) or o.get_device() != dev or o.dtype not in _DT:
                _refuse("results", o, dev)
            if o.shape != g.shape or not (g.is_contiguous() and o.is_contiguous() or o.stride() == g.stride()):
                raise ValueError("a result has the shape and strides of its gradient")
            if _DT[o.dtype] != dt and o.dtype is not _F32:
                raise ValueError("a result has the type of its gradient or float32")
        rows[1::4] = array("Q", map(_address_of, out))
        rows[3::4] = array("Q", [dt | _DT[o.dtype] << 32 for dt, o in zip(types, out)])
    else:
        rows[3::4] = array("Q", [dt | dt << 32 for dt in types])
    return rows, n


def _scalar(name, t, dev):
    if t is None:
        return None
    if t.numel() != 1 or t.dtype is not _F32 or t.get_device() != dev:
        raise ValueError(f"{name} is one float32 on the handle's device")
    return t.data_ptr()


def _call(fn, what, handle, grads, out, max_norm, inv_scale, found_inf, eps) -> Norm:
    dev = handle.device
    max_norm = math.inf if max_norm is None else float(max_norm)
    if not max_norm > 0.0 or not 0.0 <= eps < math.inf:
        raise ValueError("max_norm is positive (None: no clipping), eps is not negative")
    inv, flag = _scalar("inv_scale", inv_scale, dev), _scalar("found_inf", found_inf, dev)
    rows, n = _table(grads, out, dev)
    both = _empty((2,), (1,), dtype=_F32, device=f"cuda:{dev}")
    at = both.data_ptr()
    rc = fn(handle._h, rows.buffer_info()[0] if n else None, n, inv, max_norm, eps, at, at + 4, flag, _raw_stream(dev))
    if rc:
        handle._check(rc, what)
    return Norm(both[0], both[1])


def grad_norm(handle: stq.Handle, grads: Sequence[Optional[torch.Tensor]], *, max_norm: float | None = None,
              inv_scale: torch.Tensor | None = None, found_inf: torch.Tensor | None = None, eps: float = 1e-6, stream=None) -> Norm:
    """norm = inv_scale * 2-norm of all gradients, factor = inv_scale * min(1, max_norm / (norm + eps)).  ``inv_scale``: one float32
    on the device (1 / loss scale); ``found_inf``: one float32 on the device, set to 1 where the norm is not finite."""
    if stream is not None:
        with _On(stream, (*grads, inv_scale, found_inf)):
            return grad_norm(handle, grads, max_norm=max_norm, inv_scale=inv_scale, found_inf=found_inf, eps=eps)
    return _call((_fn or _lib()).stq_grad_norm, "stq_grad_norm", handle, grads, None, max_norm, inv_scale, found_inf, eps)


def clip_grads(handle: stq.Handle, grads: Sequence[Optional[torch.Tensor]], max_norm: float | None, *,
               inv_scale: torch.Tensor | None = None, found_inf: torch.Tensor | None = None, eps: float = 1e-6,
               out: Sequence[Optional[torch.Tensor]] | None = None, stream=None) -> Norm:
    """``grad_norm``, and the gradients times the factor: in place, or written to ``out`` (a tensor for each gradient, of its type or
    float32; the gradients stay as they are)."""
    if out is not None and len(out) != len(grads):
        raise ValueError("out has a tensor for each gradient")
    if stream is not None:
        with _On(stream, (*grads, *(out or ()), inv_scale, found_inf)):
            return clip_grads(handle, grads, max_norm, inv_scale=inv_scale, found_inf=found_inf, eps=eps, out=out)
    r = _call((_fn or _lib()).stq_grad_clip, "stq_grad_clip", handle, grads, out, max_norm, inv_scale, found_inf, eps)
    # (written behind torch's back)
    written = [t for g, t in zip(grads, grads if out is None else out) if g is not None]
    if any(map(torch.Tensor.is_inference, written)):
        written = [t for t in written if not t.is_inference()]
    torch.autograd.graph.increment_version(written)
    return r
