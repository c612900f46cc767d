"""A feed-forward block that keeps everything it saves in 8 bits, as a torch module over the operators of ``q8``.

    h   = x + residual                         (the residual stream)
    n   = rmsnorm(h) * weight                  8-bit rows
    z   = n w_in^T (+ b_in)                    8-bit product
    a   = silu(z_gate) * z_up   or   gelu(z)   8-bit rows; z itself kept as an 8-bit checkpoint
    y   = a w_out^T (+ b_out)                  8-bit product

Between the forward and the backward pass the block holds n, a and z in 8 bits (with their scales), the 8-bit weights and
h, which the stream carries anyway: per token of a gated block D + 3F + 2F/32 bytes next to h, against 2 (D + 3F) in bf16.
Gradients pass straight through the roundings.  The master weights are fp32 parameters with fp32 gradients, as
``optim.STQAdamW`` takes them.
"""
from __future__ import annotations

import math
from typing import Optional

import torch

from . import q8, stq


def _version(p: torch.Tensor):
    return None if p.is_inference() else p._version      # (how often torch has seen it change)


def _flat(t):
    """[..., width] as rows that the operators take: unit stride, no two rows in the same place."""
    if t is None:
        return None
    t = t.reshape(-1, t.shape[-1])
    return t if t.stride(1) == 1 and t.stride(0) >= t.shape[1] else t.contiguous()


class _Final(torch.autograd.Function):
    """Hands gradients on that nothing may differentiate again: the kernels that formed them leave no graph behind, and
    without this they would pass for constants.  (`anchor` requires a gradient, whatever the others do.)"""
    @staticmethod
    def forward(ctx, anchor, *grads):
        return tuple(None if g is None else g.view_as(g) for g in grads)

    @staticmethod
    def backward(ctx, *dd):
        raise RuntimeError("FeedForward8 has no second derivatives")


class _Block(torch.autograd.Function):
    @staticmethod
    def forward(ctx, block, w8, train, x, residual, weight, w_in, b_in, w_out, b_out):
        hd = block.handle_for(x.device)
        n = q8.norm(hd, x, weight, residual=residual, eps=block.eps)
        z = q8.linear(hd, n.rows, w8[0], bias=b_in)
        a = q8.act(hd, z, block.kind, checkpoint=train)
        y = q8.linear(hd, a.rows, w8[1], bias=b_out)
        if train:
            ctx.block, ck = block, a.checkpoint
            ctx.meta = ck.cols, ck.kind
            ctx.save_for_backward(n.h, n.rstd, *n.rows, *a.rows, ck.q, ck.scale, weight, *w8[0], *w8[1])
        # (an input that is returned as it is would be taken for a view of itself)
        return y, (n.h.view_as(n.h) if residual is None else n.h)

    @staticmethod
    def backward(ctx, dy, dh):
        with torch.no_grad():
            grads = _Block.gradients(ctx, dy, dh)
        if torch.is_grad_enabled():      # create_graph
            return _Final.apply(torch.empty(0, requires_grad=True), *grads)
        return grads

    @staticmethod
    def gradients(ctx, dy, dh):
        h, rstd, nq, ns, aq, as_, cq, cs, weight, iq, is_, oq, os_ = ctx.saved_tensors
        hd = ctx.block.ordered_handle(h.device)
        dy, dh = dy.contiguous(), dh.contiguous()
        rows8 = q8.Rows8
        _, _, _, for_x, for_res, for_weight, for_w_in, for_b_in, for_w_out, for_b_out = ctx.needs_input_grad
        dx = dweight = dw_in = db_in = dw_out = db_out = None      # (formed only if somebody asks)
        if for_w_out:
            dw_out = q8.linear_dw(hd, dy, rows8(aq, as_), dtype=torch.float32)
        if for_b_out:
            db_out = q8.bias_grad(hd, dy)
        before_z = for_x or for_res or for_weight
        if before_z or for_w_in or for_b_in:
            dz = q8.act_backward(hd, q8.linear_dx(hd, dy, rows8(oq, os_)), q8.Checkpoint8(cq, cs, *ctx.meta))
            if for_w_in:
                dw_in = q8.linear_dw(hd, dz, rows8(nq, ns), dtype=torch.float32)
            if for_b_in:
                db_in = q8.bias_grad(hd, dz)
            if before_z:
                dx, dweight = q8.norm_backward(hd, q8.linear_dx(hd, dz, rows8(iq, is_)), h, weight, rstd, dres=dh)
        return (None, None, None, dx if for_x else None, dx if for_res else None, dweight if for_weight else None, dw_in,
                db_in, dw_out, db_out)


class FeedForward8(torch.nn.Module):
    """norm -> product -> activation -> product, with 8-bit products and 8-bit saved state.

    forward(x, residual=None) takes bf16 [..., width] in any layout and returns (y, h) with h = x + residual: the next block
    of a stack gets them as its x and residual.  kind: "silu_gated" or "gelu".  In training the weights are quantized on
    every forward pass (an optimizer step has changed them); ``freeze()`` quantizes them once, for serving under
    ``torch.no_grad()``.  A frozen block quantizes them again where they have changed since (loading, an optimizer step, any
    change that torch counts, a move to another device), and for every pass that differentiates them.  There are no second
    derivatives: differentiating the gradients raises.

    Passes may run on any streams: backward passes, which share a workspace, are put in order one after the other.  A
    captured graph that holds a backward pass must not be replayed while another backward pass of the block runs."""

    def __init__(self, width: int, hidden: int, kind: str = "silu_gated", bias: bool = False, eps: float = 1e-6, device="cuda"):
        super().__init__()
        if kind not in q8.KINDS:
            raise ValueError("kind is one of " + ", ".join(q8.KINDS))
        self.kind, self.eps = kind, float(eps)
        parts = 2 if kind == "silu_gated" else 1
        new = lambda *s: torch.nn.Parameter(torch.empty(*s, dtype=torch.float32, device=device))  # noqa: E731
        self.weight = torch.nn.Parameter(torch.ones(width, dtype=torch.float32, device=device))
        self.w_in, self.w_out = new(parts * hidden, width), new(width, hidden)
        torch.nn.init.normal_(self.w_in, std=1 / math.sqrt(width))
        torch.nn.init.normal_(self.w_out, std=1 / math.sqrt(hidden))
        self.b_in = torch.nn.Parameter(torch.zeros(parts * hidden, dtype=torch.float32, device=device)) if bias else None
        self.b_out = torch.nn.Parameter(torch.zeros(width, dtype=torch.float32, device=device)) if bias else None
        self.weights8 = None
        self._of = None        # what weights8 was quantized from: the parameters, their versions, on which stream and when
        self._in_graphs = []   # codes that captured graphs read
        self._handle: Optional[stq.Handle] = None
        self._last = None      # the stream of the last backward pass

    def handle_for(self, device: torch.device) -> stq.Handle:
        if self._handle is None or self._handle.device != device.index:
            self._handle, self._last = stq.Handle(device.index), None
        return self._handle

    def ordered_handle(self, device: torch.device) -> stq.Handle:
        """The handle for a backward pass on the current stream.  Backward calls share the handle's workspace, so the stream
        waits for the one of the last backward pass.  (A capture runs nothing: who replays the graph keeps the order.)"""
        hd = self.handle_for(device)
        if not torch.cuda.is_current_stream_capturing():
            stream = torch.cuda.current_stream(device)
            if self._last is not None and self._last != stream:
                stream.wait_stream(self._last)
            self._last = stream
        return hd

    def __getstate__(self):
        # (a copy makes its own, and quantizes its own weights)
        return {**self.__dict__, "_handle": None, "_last": None, "_of": None, "_in_graphs": []}

    def quantized(self):
        """The two weights as 8-bit rows, a scale per output channel."""
        hd = self.handle_for(self.w_in.device)
        return q8.quantize_rows(hd, self.w_in.detach()), q8.quantize_rows(hd, self.w_out.detach())

    def freeze(self):
        """Quantizes the weights once and keeps them until ``thaw()``: for serving, where they do not change."""
        with torch.inference_mode(False):      # (a later pass may have to save them)
            self.weights8 = self.quantized()
        self._of = None
        if not torch.cuda.is_current_stream_capturing():      # (a capture has not computed anything yet)
            stream, done = torch.cuda.current_stream(self.w_in.device), torch.cuda.Event()
            done.record(stream)
            self._of = self.w_in, _version(self.w_in), self.w_out, _version(self.w_out), stream.cuda_stream, done
        return self

    def thaw(self):
        self.weights8 = self._of = None
        return self

    def _codes(self, differentiated: bool):
        """The 8-bit weights for a pass on the current stream."""
        if self.weights8 is None:
            return self.quantized()
        if differentiated:      # they are about to change, by an optimizer that may write them behind torch's back
            self._of = None
            return self.quantized()
        of, capturing = self._of, torch.cuda.is_current_stream_capturing()
        w_in, w_out = self.w_in, self.w_out
        if of is None or of[0] is not w_in or of[1] != _version(w_in) or of[2] is not w_out or of[3] != _version(w_out):
            if capturing:       # (every replay quantizes)
                return self.quantized()
            self.freeze()
        elif capturing:         # the graph goes on reading them, whatever the block serves by then
            if all(c is not self.weights8 for c in self._in_graphs):
                self._in_graphs.append(self.weights8)
        elif of[4] != q8._raw_stream(w_in.device.index):      # another stream than the one that wrote them
            stream = torch.cuda.current_stream(w_in.device)
            stream.wait_event(of[5])
            for r in self.weights8:
                r.q.record_stream(stream), r.scale.record_stream(stream)
        return self.weights8

    def _apply(self, *args, **kw):
        self._of = None            # (parameters that move or change their type keep their version)
        return super()._apply(*args, **kw)

    def _load_from_state_dict(self, *args, **kw):
        self._of = None
        return super()._load_from_state_dict(*args, **kw)

    def saved_bytes(self, tokens: int) -> int:
        """Bytes that a forward pass of so many tokens keeps for its backward pass, next to h and the weights."""
        (hidden, width), up = self.w_out.t().shape, lambda n: (n + 15) // 16 * 16
        parts = self.w_in.shape[0] // hidden
        return tokens * (up(width) + up(hidden) + parts * (up(hidden) + 4 * -(-hidden // q8.CKPT_BLOCK)) + 12)

    def forward(self, x: torch.Tensor, residual: torch.Tensor | None = None):
        if x.dtype != torch.bfloat16 or (residual is not None and residual.dtype != torch.bfloat16):
            raise ValueError("FeedForward8 takes bfloat16 activations")
        given = (_flat(x), _flat(residual), self.weight, self.w_in, self.b_in, self.w_out, self.b_out)
        # (inside a Function neither the grad mode nor needs_input_grad tells whether a backward pass can follow)
        train = torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in given)
        w8 = self._codes(train and (self.w_in.requires_grad or self.w_out.requires_grad))
        y, h = _Block.apply(self, w8, train, *given)
        return y.view(x.shape), h.view(x.shape)
