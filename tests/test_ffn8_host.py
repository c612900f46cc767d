"""The feed-forward block's order of work on the host (no GPU: streams and handles are stand-ins)."""
import copy
from types import SimpleNamespace

import pytest
import torch

from paper_2604_06836_b200 import ffn8


class Stream:
    def __init__(self, name, log):
        self.name, self.log = name, log

    def wait_stream(self, other):
        self.log.append((self.name, other.name))


@pytest.fixture
def cuda(monkeypatch):
    """Stand-ins for what the block asks of torch and the library: `now` is the current stream."""
    state = SimpleNamespace(log=[], now=None, capturing=False, handles=0)

    def handle(index):
        state.handles += 1
        return SimpleNamespace(device=index)
    monkeypatch.setattr(ffn8.stq, "Handle", handle)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: state.now)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state.capturing)
    state.stream = lambda name: Stream(name, state.log)
    return state


# ---- streams -----------------------------------------------------------------------------------------------------------
def test_backward_passes_on_different_streams_are_put_in_order(cuda):
    m, dev = ffn8.FeedForward8(16, 32, device="cpu"), SimpleNamespace(index=0)
    a, b, c = (cuda.stream(n) for n in "abc")
    for s in (a, a, b, b, a):
        cuda.now = s
        hd = m.ordered_handle(dev)
        assert hd is m.handle_for(dev)
    assert cuda.log == [("b", "a"), ("a", "b")] and cuda.handles == 1
    cuda.capturing, cuda.now = True, c                    # a capture neither waits nor is waited for
    m.ordered_handle(dev)
    cuda.capturing, cuda.now = False, b
    m.ordered_handle(dev)
    assert cuda.log == [("b", "a"), ("a", "b"), ("b", "a")]
    twin = copy.deepcopy(m)                               # a copy has a workspace of its own
    cuda.now = a
    twin.ordered_handle(dev)
    assert len(cuda.log) == 3 and cuda.handles == 2
    m.ordered_handle(SimpleNamespace(index=1))            # so has the block on another device
    assert len(cuda.log) == 3 and cuda.handles == 3
