"""The last layer of a language model or classifier, with its loss, as a torch module over the operators of ``vocab``.

    loss[i] = log sum_j exp z[i][j] - z[i][target[i]],   z = h weight^T (+ bias)

The logits are never kept, neither for the backward pass nor between the two: a batch of 8192 tokens over 50257 entries would hold
1.6 GB of them in fp32.  The master weight is an fp32 parameter with an fp32 gradient, as ``optim.STQAdamW`` takes it (or a bf16
one with a bf16 gradient); the products take it rounded to bf16.
"""
from __future__ import annotations

import math
from typing import Optional

import torch

from . import q8, stq, vocab
from .ffn8 import _flat


class _Final(torch.autograd.Function):
    """Hands gradients on that nothing may differentiate again (the kernels that formed them leave no graph behind)."""
    @staticmethod
    def forward(ctx, anchor, *grads):
        return tuple(None if g is None else g.view_as(g) for g in grads)

    @staticmethod
    def backward(ctx, *dd):
        raise RuntimeError("VocabLoss has no second derivatives")


class _Loss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, head, x, weight, bias, target):
        w = weight if weight.dtype == torch.bfloat16 else weight.to(torch.bfloat16)
        out = vocab.loss(head.ordered_handle(x.device), x, w, target, bias=bias, ignore_index=head.ignore_index)
        ctx.head, ctx.dtype, ctx.ignore_index = head, weight.dtype, head.ignore_index
        ctx.save_for_backward(x, w, bias, target, out.lse)
        ctx.mark_non_differentiable(out.lse)
        return out.loss, out.lse

    @staticmethod
    def backward(ctx, dloss, _):
        x, w, bias, target, lse = ctx.saved_tensors
        _, for_x, for_w, for_b, _ = ctx.needs_input_grad
        with torch.no_grad():
            g = vocab.loss_backward(ctx.head.ordered_handle(x.device), dloss.contiguous(), x, w, target, lse, bias=bias,
                                    ignore_index=ctx.ignore_index, dtype=ctx.dtype, want_dx=for_x, want_dw=for_w, want_dbias=for_b)
        grads = g.dx, g.dw, g.dbias
        if torch.is_grad_enabled():      # create_graph
            grads = _Final.apply(torch.empty(0, requires_grad=True), *grads)
        return None, *grads, None


class VocabLoss(torch.nn.Module):
    """Output matrix and cross entropy.

    forward(h, target, reduction="mean") takes bf16 hidden states [..., width] in any layout and int64 targets [...], and returns the
    mean over the tokens that count (0 if none does), their "sum", or the loss of each token ("none", float32 [...]).  ``scores``
    gives the log probability of each target, for serving: nothing is saved.  weight: an existing parameter [vocab, width] (tied to
    an embedding), else a new one.  The weight is rounded to bf16 in every pass; ``freeze()`` rounds it once, for serving under
    ``torch.no_grad()``, until ``thaw()`` or until torch counts a change of it.  There are no second derivatives.

    Passes may run on any streams: they share a workspace and are put in order one after the other.  A captured graph that holds a
    pass must not be replayed while another pass of the module runs; and, as with every module, no loss of an eager pass over the same
    parameters may be alive while a backward pass is captured (torch would order the capture behind that pass's stream)."""

    def __init__(self, width: int, vocab: int, bias: bool = False, ignore_index: int = -100,
                 weight: Optional[torch.nn.Parameter] = None, device="cuda"):
        super().__init__()
        if weight is None:
            weight = torch.nn.Parameter(torch.empty(vocab, width, dtype=torch.float32, device=device))
            torch.nn.init.normal_(weight, std=1 / math.sqrt(width))
        elif tuple(weight.shape) != (vocab, width) or weight.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError(f"weight is float32 or bfloat16 [{vocab}, {width}]")
        self.weight, self.ignore_index = weight, int(ignore_index)
        self.bias = torch.nn.Parameter(torch.zeros(vocab, dtype=torch.float32, device=weight.device)) if bias else None
        self._handle: Optional[stq.Handle] = None
        self._last = None        # the stream of the last pass
        self._kept = None        # frozen: the rounded weight, what it was rounded from, and when it was ready on which stream
        self._frozen = False
        self._in_graphs = []     # rounded weights that captured graphs read

    def ordered_handle(self, device: torch.device) -> stq.Handle:
        """The handle for a pass on the current stream, which waits for the stream of the last pass.  (A capture runs nothing: who
        replays the graph keeps the order.)"""
        if self._handle is None or self._handle.device != device.index:
            self._handle, self._last = stq.Handle(device.index), None
        if not torch.cuda.is_current_stream_capturing():
            stream = torch.cuda.current_stream(device)
            if self._last is not None and self._last != stream:
                stream.wait_stream(self._last)
            self._last = stream
        return self._handle

    def __getstate__(self):
        return {**self.__dict__, "_handle": None, "_last": None, "_kept": None, "_in_graphs": []}

    def freeze(self):
        self._frozen, self._kept = True, None
        return self

    def thaw(self):
        self._frozen, self._kept = False, None
        return self

    def _apply(self, *args, **kw):
        self._kept = None
        return super()._apply(*args, **kw)

    def _load_from_state_dict(self, *args, **kw):
        self._kept = None
        return super()._load_from_state_dict(*args, **kw)

    def _served(self):
        """The weight in bf16 for a pass that nothing differentiates."""
        w = self.weight.detach()
        if w.dtype == torch.bfloat16:
            return w
        if not self._frozen or self.weight.is_inference():
            return w.to(torch.bfloat16)
        capturing = torch.cuda.is_current_stream_capturing()
        kept, version = self._kept, self.weight._version
        if kept is None or kept[1] is not self.weight or kept[2] != version:
            with torch.inference_mode(False):
                rounded = w.to(torch.bfloat16)
            if not capturing:      # (a capture has not computed anything yet: every replay rounds)
                stream, done = torch.cuda.current_stream(w.device), torch.cuda.Event()
                done.record(stream)
                self._kept = rounded, self.weight, version, stream.cuda_stream, done
            return rounded
        if capturing:              # the graph goes on reading it, whatever is served by then
            if all(k is not kept[0] for k in self._in_graphs):
                self._in_graphs.append(kept[0])
        elif kept[3] != q8._raw_stream(w.device.index):
            stream = torch.cuda.current_stream(w.device)
            stream.wait_event(kept[4])
            kept[0].record_stream(stream)
        return kept[0]

    def _checked(self, h, target):
        if h.dtype != torch.bfloat16:
            raise ValueError("VocabLoss takes bfloat16 hidden states")
        if target.shape != h.shape[:-1]:
            raise ValueError("there is a target for each hidden state")
        return _flat(h), target.reshape(-1).contiguous()

    @torch.no_grad()
    def scores(self, h: torch.Tensor, target: torch.Tensor) -> torch.Tensor:
        """Log probability of each target (0 where it is ignore_index)."""
        x, to = self._checked(h, target)
        w = self._served()
        out = vocab.loss(self.ordered_handle(x.device), x, w, to, bias=None if self.bias is None else self.bias.detach(),
                         ignore_index=self.ignore_index)
        return out.loss.neg_().view(target.shape)

    def forward(self, h: torch.Tensor, target: torch.Tensor, reduction: str = "mean") -> torch.Tensor:
        if reduction not in ("mean", "sum", "none"):
            raise ValueError("reduction is mean, sum or none")
        x, to = self._checked(h, target)
        given = (x, self.weight, self.bias)
        if torch.is_grad_enabled() and any(p is not None and p.requires_grad for p in given):
            loss, _ = _Loss.apply(self, *given, to)
        else:
            loss = -self.scores(h, target).reshape(-1)
        if reduction == "none":
            return loss.view(target.shape)
        if reduction == "sum":
            return loss.sum()
        return loss.sum() / (to != self.ignore_index).sum().clamp(min=1)
