"""8-bit operators of a feed-forward block: a root-mean-square norm and an activation that write 8-bit rows, the
product of 8-bit rows with 8-bit weights, and their gradients, which read what the forward pass saved in 8 bits.

Thin binding over the ``stq_q8_*`` calls of libstq, like ``stq``: torch supplies memory and streams, every
operator runs in the library's kernels.  All matrices are two-dimensional with unit stride along a row; any row pitch
is taken.  Each call enqueues its work on the current stream of the handle's device (or on ``stream``) and does not
synchronise, except where a backward call needs more workspace than any before it (the old one is then freed).  One
handle serves one stream at a time: its workspace is shared by the calls made through it, and by the graphs captured
with it, which stay valid as long as the handle does.  Once a wait inside a kernel has run out (its results are invalid
then), the handle's next call raises StqError with code -11; ``Handle.device_status()`` synchronises and asks.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional

import torch

from . import stq

_F32, _BF16, _I8 = torch.float32, torch.bfloat16, torch.int8
_empty = torch.empty_strided
CKPT_BLOCK = 128                                   # STQ_CKPT_BLOCK: columns per scale of a checkpoint
KINDS = {"silu_gated": 1, "gelu": 2}               # STQ_ACT_*
_DTYPES = {torch.float32: stq.GRAD_F32, torch.bfloat16: stq.GRAD_BF16}
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda dev: torch.cuda.current_stream(dev).cuda_stream)      # (a build of torch without CUDA)

_fn = None


def _lib() -> C.CDLL:
    global _fn
    if _fn is None:
        L = stq.lib()
        vp, u64, u32, i, f = C.c_void_p, C.c_uint64, C.c_uint32, C.c_int, C.c_float
        L.stq_q8_rows.argtypes = [vp, vp, u64, i, u64, u32, vp, u64, vp, vp]
        L.stq_q8_norm.argtypes = [vp, vp, u64, vp, u64, vp, f, i, u64, u32, vp, u64, vp, vp, u64, vp, vp, u64, vp]
        L.stq_q8_norm_backward.argtypes = [vp, vp, u64, vp, u64, vp, vp, vp, u64, i, u64, u32, vp, u64, vp, vp]
        L.stq_q8_act.argtypes = [vp, vp, u64, i, i, u64, u32, vp, u64, vp, vp, u64, vp, u64, vp, vp]
        L.stq_q8_act_backward.argtypes = [vp, vp, u64, i, i, u64, u32, vp, u64, vp, vp, u64, vp]
        L.stq_q8_linear.argtypes = [vp, vp, u64, vp, vp, u64, vp, vp, u64, u32, u32, vp, u64, i, vp]
        L.stq_q8_linear_dx.argtypes = [vp, vp, u64, vp, u64, vp, u64, u32, u32, vp, u64, i, vp]
        L.stq_q8_linear_dw.argtypes = [vp, vp, u64, vp, u64, vp, u64, u32, u32, vp, u64, i, vp]
        L.stq_q8_bias_grad.argtypes = [vp, vp, u64, i, u64, u32, vp, vp]
        _fn = L
    return _fn


class Rows8(NamedTuple):
    """8-bit rows: value = q * scale[row].  q: int8 [rows, cols], row pitch a multiple of 16 bytes."""
    q: torch.Tensor
    scale: torch.Tensor

    def values(self, dtype=torch.float32) -> torch.Tensor:
        """The values that the codes stand for (plain torch arithmetic, for inspection)."""
        return (self.q.float() * self.scale[:, None]).to(dtype)


class Checkpoint8(NamedTuple):
    """The input of an activation in 8 bits, one scale per CKPT_BLOCK columns.  q: int8 [rows, parts, pitch], scale:
    float32 [rows, parts, blocks]."""
    q: torch.Tensor
    scale: torch.Tensor
    cols: int
    kind: str

    def nbytes(self) -> int:
        return self.q.numel() + 4 * self.scale.numel()

    def values(self) -> torch.Tensor:
        """The saved input as float32 [rows, parts * cols] (plain torch arithmetic, for inspection)."""
        s = self.scale.repeat_interleave(CKPT_BLOCK, dim=2)[:, :, :self.cols]
        return (self.q[:, :, :self.cols].float() * s).reshape(self.q.shape[0], -1)


class NormOut(NamedTuple):
    h: torch.Tensor                  # x + residual (x itself without a residual)
    rows: Rows8                      # the norm of h in 8 bits
    rstd: torch.Tensor               # float32 [rows]
    values: Optional[torch.Tensor]   # bf16 values of `rows`, if asked for


class ActOut(NamedTuple):
    rows: Rows8
    checkpoint: Optional[Checkpoint8]
    values: Optional[torch.Tensor]


# ---- arguments ---------------------------------------------------------------------------------------------------
# The checks run on every call, also for a single token, so the usual case takes as few steps as it can; what is wrong
# is found out only once something is.
def _pitch(t: torch.Tensor, dev: int, dtype, rows, cols) -> int:
    """Row pitch in elements of a matrix that is as it should be (None: anything goes), else -1."""
    shape = t.shape
    if len(shape) != 2 or t.get_device() != dev or (dtype is not None and t.dtype is not dtype):
        return -1
    r, c = shape
    if (rows is not None and r != rows) or (cols is not None and c != cols):
        return -1
    ld, unit = t.stride()
    if unit != 1 and c > 1:
        return -1
    if ld < c:
        return c if r <= 1 else -1
    return ld


def _refuse(name: str, t: torch.Tensor, dev: int, dtype, rows, cols):
    if t.dim() != 2:
        raise ValueError(f"{name} is a matrix")
    if t.get_device() != dev:
        raise ValueError(f"{name} lives on the handle's device")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} is {dtype}, not {t.dtype}")
    r, c = t.shape
    if rows is not None and r != rows:
        raise ValueError(f"{name} has {rows} rows, not {r}")
    if cols is not None and c != cols:
        raise ValueError(f"{name} has {cols} columns, not {c}")
    if t.stride(1) != 1 and c > 1:
        raise ValueError(f"{name} has unit stride along a row")
    raise ValueError(f"{name}'s rows do not overlap")


def _mat(name: str, t: torch.Tensor, dev: int, dtype=None, rows=None, cols=None) -> int:
    ld = _pitch(t, dev, dtype, rows, cols)
    if ld < 0:
        _refuse(name, t, dev, dtype, rows, cols)
    return ld


def _vec(name: str, t: torch.Tensor, dev: int, n: int):
    if t.shape != (n,) or t.dtype is not _F32 or not t.is_contiguous():
        raise ValueError(f"{name} is a contiguous float32 vector of {n}")
    if t.get_device() != dev:
        raise ValueError(f"{name} lives on the handle's device")


def _rows(name: str, r: Rows8, dev: int, cols=None, rows=None) -> int:
    q, scale = r
    ld = _pitch(q, dev, _I8, rows, cols)
    if ld < 0:
        _refuse(name + ".q", q, dev, _I8, rows, cols)
    n = q.shape[0]
    _vec(name + ".scale", scale, dev, n)
    return (ld + 15) & ~15 if n <= 1 else ld


def _dtype(name: str, t: torch.Tensor) -> int:
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        raise ValueError(f"{name} is float32 or bfloat16, not {t.dtype}")
    return dt


def _out_dtype(dtype) -> int:
    dt = _DTYPES.get(dtype)
    if dt is None:
        raise ValueError(f"dtype is float32 or bfloat16, not {dtype}")
    return dt


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


class _On:
    """Work on a stream other than the current one: outputs are allocated there, and the allocator is told that the
    inputs are in use there."""

    def __init__(self, stream, inputs):
        self._ctx = torch.cuda.stream(stream)
        for t in inputs:
            if t is not None:
                t.record_stream(stream)

    def __enter__(self):
        self._ctx.__enter__()

    def __exit__(self, *a):
        self._ctx.__exit__(*a)


def _new(rows: int, cols: int, pitch: int, dtype, device) -> torch.Tensor:
    return _empty((rows, cols), (pitch, 1), dtype=dtype, device=device)


def _new_vec(n: int, device) -> torch.Tensor:
    return _empty((n,), (1,), dtype=_F32, device=device)


def alloc_rows(rows: int, cols: int, device) -> Rows8:
    """Uninitialised 8-bit rows with the pitch that the operators need."""
    return Rows8(_new(rows, cols, (cols + 15) // 16 * 16, torch.int8, device), _new_vec(rows, device))


# ---- operators ---------------------------------------------------------------------------------------------------
def quantize_rows(handle: stq.Handle, x: torch.Tensor, *, out: Rows8 | None = None, stream=None) -> Rows8:
    """x [rows, cols] in 8 bits with a scale per row (for a weight [out, in]: per output channel)."""
    if stream is not None:
        with _On(stream, (x,) + (tuple(out) if out is not None else ())):
            return quantize_rows(handle, x, out=out)
    dev = handle.device
    dt, ldx = _dtype("x", x), _mat("x", x, dev)
    rows, cols = x.shape
    if out is None:
        out = alloc_rows(rows, cols, x.device)
    ldq = _rows("out", out, dev, cols, rows)
    rc = (_fn or _lib()).stq_q8_rows(handle._h, x.data_ptr(), ldx, dt, rows, cols, out.q.data_ptr(), ldq,
        out.scale.data_ptr(), _raw_stream(dev))
    if rc:
        handle._check(rc, "stq_q8_rows")
    return out


def norm(handle: stq.Handle, x: torch.Tensor, weight: torch.Tensor, *, residual: torch.Tensor | None = None,
         eps: float = 1e-6, values: bool = False, stream=None) -> NormOut:
    """h = x + residual; its root-mean-square norm times weight, as 8-bit rows.  weight: float32 [cols]."""
    if stream is not None:
        with _On(stream, (x, weight, residual)):
            return norm(handle, x, weight, residual=residual, eps=eps, values=values)
    dev = handle.device
    kind = x.dtype
    dt, ldx = _dtype("x", x), _mat("x", x, dev)
    rows, cols = x.shape
    _vec("weight", weight, dev, cols)
    device, pitch = x.device, (cols + 15) & ~15
    h, res_ptr, ldres, h_ptr = x, None, 0, None
    if residual is not None:
        ldres = _mat("residual", residual, dev, kind, rows, cols)
        h = _empty((rows, cols), (cols, 1), dtype=kind, device=device)
        res_ptr, h_ptr = residual.data_ptr(), h.data_ptr()
    q = _empty((rows, cols), (pitch, 1), dtype=_I8, device=device)
    scale = _empty((rows,), (1,), dtype=_F32, device=device)
    stats = _empty((rows,), (1,), dtype=_F32, device=device)
    vals, v_ptr = None, None
    if values:
        vals = _empty((rows, cols), (cols, 1), dtype=_BF16, device=device)
        v_ptr = vals.data_ptr()
    rc = (_fn or _lib()).stq_q8_norm(
        handle._h, x.data_ptr(), ldx, res_ptr, ldres, weight.data_ptr(), eps, dt, rows, cols, h_ptr, cols,
        stats.data_ptr(), q.data_ptr(), pitch, scale.data_ptr(), v_ptr, cols, _raw_stream(dev))
    if rc:
        handle._check(rc, "stq_q8_norm")
    return NormOut(h, Rows8(q, scale), stats, vals)


def norm_backward(handle: stq.Handle, dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor, rstd: torch.Tensor, *,
                  dres: torch.Tensor | None = None, stream=None):
    """(dx, dweight) of ``norm``; dx is the gradient of x and of the residual alike, with ``dres`` (what reaches h from
    elsewhere) added.  dweight is float32."""
    if stream is not None:
        with _On(stream, (dy, h, weight, rstd, dres)):
            return norm_backward(handle, dy, h, weight, rstd, dres=dres)
    dev = handle.device
    dt, lddy = _dtype("dy", dy), _mat("dy", dy, dev)
    rows, cols = dy.shape
    ldh = _mat("h", h, dev, dy.dtype, rows, cols)
    _vec("weight", weight, dev, cols)
    _vec("rstd", rstd, dev, rows)
    ldres = 0 if dres is None else _mat("dres", dres, dev, dy.dtype, rows, cols)
    dx = _new(rows, cols, cols, dy.dtype, dy.device)
    dweight = _new_vec(cols, dy.device)
    rc = (_fn or _lib()).stq_q8_norm_backward(
        handle._h, dy.data_ptr(), lddy, h.data_ptr(), ldh, weight.data_ptr(), rstd.data_ptr(),
        None if dres is None else dres.data_ptr(), ldres, dt, rows, cols, dx.data_ptr(), cols, dweight.data_ptr(),
        _raw_stream(dev))
    if rc:
        handle._check(rc, "stq_q8_norm_backward")
    return dx, dweight


def act(handle: stq.Handle, z: torch.Tensor, kind: str = "silu_gated", *, checkpoint: bool = False, values: bool = False,
        stream=None) -> ActOut:
    """silu(z[:, :f]) * z[:, f:] ("silu_gated", z [rows, 2f]) or gelu(z) ("gelu", tanh form) as 8-bit rows; with
    ``checkpoint`` z itself is kept in 8 bits for ``act_backward``."""
    if stream is not None:
        with _On(stream, (z,)):
            return act(handle, z, kind, checkpoint=checkpoint, values=values)
    if kind not in KINDS:
        raise ValueError("kind is one of " + ", ".join(KINDS))
    dev = handle.device
    dt, ldz = _dtype("z", z), _mat("z", z, dev)
    parts = 2 if kind == "silu_gated" else 1
    rows, cols = z.shape[0], z.shape[1] // parts
    _need(cols * parts == z.shape[1], "a gated activation takes an even number of columns")
    device, pitch = z.device, (cols + 15) & ~15
    q = _empty((rows, cols), (pitch, 1), dtype=_I8, device=device)
    scale = _empty((rows,), (1,), dtype=_F32, device=device)
    vals, v_ptr, ck, ckq, cks = None, None, None, None, None
    if values:
        vals = _empty((rows, cols), (cols, 1), dtype=_BF16, device=device)
        v_ptr = vals.data_ptr()
    if checkpoint:
        ck = Checkpoint8(torch.empty((rows, parts, pitch), dtype=_I8, device=device),
                         torch.empty((rows, parts, -(-cols // CKPT_BLOCK)), dtype=_F32, device=device), cols, kind)
        ckq, cks = ck.q.data_ptr(), ck.scale.data_ptr()
    rc = (_fn or _lib()).stq_q8_act(handle._h, z.data_ptr(), ldz, KINDS[kind], dt, rows, cols, q.data_ptr(), pitch,
                                    scale.data_ptr(), v_ptr, cols, ckq, pitch, cks, _raw_stream(dev))
    if rc:
        handle._check(rc, "stq_q8_act")
    return ActOut(Rows8(q, scale), ck, vals)


def act_backward(handle: stq.Handle, da: torch.Tensor, checkpoint: Checkpoint8, *, stream=None) -> torch.Tensor:
    """Gradient of the activation's input, taken at the checkpointed input."""
    if stream is not None:
        with _On(stream, (da, checkpoint.q, checkpoint.scale)):
            return act_backward(handle, da, checkpoint)
    dev = handle.device
    q, scale, cols, kind = checkpoint
    rows, parts, pitch = q.shape
    _need(kind in KINDS and parts == (2 if kind == "silu_gated" else 1), "the checkpoint's parts fit its kind")
    _need(q.dtype == torch.int8 and scale.dtype == torch.float32 and q.is_contiguous() and scale.is_contiguous()
          and scale.shape == (rows, parts, -(-cols // CKPT_BLOCK)), "the checkpoint is as act() made it")
    _need(q.device.index == dev and scale.device.index == dev and q.is_cuda and scale.is_cuda,
          "the checkpoint lives on the handle's device")
    dt, ldda = _dtype("da", da), _mat("da", da, dev, None, rows, cols)
    dz = _new(rows, parts * cols, parts * cols, da.dtype, da.device)
    rc = (_fn or _lib()).stq_q8_act_backward(handle._h, da.data_ptr(), ldda, KINDS[kind], dt, rows, cols, q.data_ptr(),
        pitch, scale.data_ptr(), dz.data_ptr(), parts * cols, _raw_stream(dev))
    if rc:
        handle._check(rc, "stq_q8_act_backward")
    return dz


def linear(handle: stq.Handle, x: Rows8, w: Rows8, *, bias: torch.Tensor | None = None, dtype=torch.bfloat16,
           stream=None) -> torch.Tensor:
    """x [t, k] times w [n, k] transposed, in 8-bit integers, with both rows' scales; plus bias (float32 [n])."""
    if stream is not None:
        with _On(stream, (*x, *w, bias)):
            return linear(handle, x, w, bias=bias, dtype=dtype)
    dev = handle.device
    odt, ldx = _out_dtype(dtype), _rows("x", x, dev)
    (xq, xs), (wq, ws) = x, w
    t, k = xq.shape
    ldw = _rows("w", w, dev, k)
    n = wq.shape[0]
    if bias is not None:
        _vec("bias", bias, dev, n)
    out = _empty((t, n), (n, 1), dtype=dtype, device=xq.device)
    rc = (_fn or _lib()).stq_q8_linear(
        handle._h, xq.data_ptr(), ldx, xs.data_ptr(), wq.data_ptr(), ldw, ws.data_ptr(),
        None if bias is None else bias.data_ptr(), t, n, k, out.data_ptr(), n, odt, _raw_stream(dev))
    if rc:
        handle._check(rc, "stq_q8_linear")
    return out


def linear_dx(handle: stq.Handle, dy: torch.Tensor, w: Rows8, *, dtype=torch.bfloat16, stream=None) -> torch.Tensor:
    """Gradient of ``linear``'s input: dy [t, n] (bfloat16) times the values of w [n, k].  For a bfloat16 result the values
    are rounded to bfloat16 on the way, with float32 they are not."""
    if stream is not None:
        with _On(stream, (dy, *w)):
            return linear_dx(handle, dy, w, dtype=dtype)
    dev = handle.device
    odt, ldw = _out_dtype(dtype), _rows("w", w, dev)
    n, k = w.q.shape
    lddy = _mat("dy", dy, dev, torch.bfloat16, None, n)
    t = dy.shape[0]
    out = _new(t, k, k, dtype, dy.device)
    rc = (_fn or _lib()).stq_q8_linear_dx(handle._h, dy.data_ptr(), lddy, w.q.data_ptr(), ldw, w.scale.data_ptr(), t, n, k,
        out.data_ptr(), k, odt, _raw_stream(dev))
    if rc:
        handle._check(rc, "stq_q8_linear_dx")
    return out


def linear_dw(handle: stq.Handle, dy: torch.Tensor, x: Rows8, *, dtype=torch.bfloat16, stream=None) -> torch.Tensor:
    """Gradient of ``linear``'s weight from its input as it was saved in 8 bits: dy [t, n] (bfloat16) transposed times
    the values of x [t, k].  For a bfloat16 result the values are rounded to bfloat16 on the way, with float32 they are not."""
    if stream is not None:
        with _On(stream, (dy, *x)):
            return linear_dw(handle, dy, x, dtype=dtype)
    dev = handle.device
    odt, ldx = _out_dtype(dtype), _rows("x", x, dev)
    t, k = x.q.shape
    lddy = _mat("dy", dy, dev, torch.bfloat16, t)
    n = dy.shape[1]
    out = _new(n, k, k, dtype, dy.device)
    rc = (_fn or _lib()).stq_q8_linear_dw(handle._h, dy.data_ptr(), lddy, x.q.data_ptr(), ldx, x.scale.data_ptr(), t, n, k,
        out.data_ptr(), k, odt, _raw_stream(dev))
    if rc:
        handle._check(rc, "stq_q8_linear_dw")
    return out


def bias_grad(handle: stq.Handle, dy: torch.Tensor, *, stream=None) -> torch.Tensor:
    """Gradient of a bias: the column sums of dy, float32."""
    if stream is not None:
        with _On(stream, (dy,)):
            return bias_grad(handle, dy)
    dev = handle.device
    dt, ld = _dtype("dy", dy), _mat("dy", dy, dev)
    t, n = dy.shape
    out = _new_vec(n, dy.device)
    rc = (_fn or _lib()).stq_q8_bias_grad(handle._h, dy.data_ptr(), ld, dt, t, n, out.data_ptr(), _raw_stream(dev))
    if rc:
        handle._check(rc, "stq_q8_bias_grad")
    return out
