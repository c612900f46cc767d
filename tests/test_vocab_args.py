"""The vocabulary cross entropy and the gradient norm refuse what they cannot take before anything reaches a device (no GPU)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2604_06836_b200 import clip, vocab
from paper_2604_06836_b200.head import VocabLoss

HANDLE = SimpleNamespace(device=0, _h=None)      # (no call below gets as far as using it)
X, W, T = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(9, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)


@pytest.mark.parametrize("call,what", [
    (lambda: vocab.loss(HANDLE, X, W, T), "device"),
    (lambda: vocab.loss(HANDLE, X[0], W, T), "matrix"),
    (lambda: vocab.loss_backward(HANDLE, T.float(), X, W, T, T.float()), "device"),
    (lambda: vocab.loss_backward(HANDLE, T.float(), X, W, T, T.float(), dtype=torch.float16), "float32 or bfloat16"),
    (lambda: vocab._targets(T, -1, 5), "int64 vector of 5"),
    (lambda: vocab._targets(T.int(), -1, 4), "int64"),
    (lambda: vocab._targets(T[::2], -1, 2), "contiguous"),
    (lambda: vocab._targets(T, 0, 4), "device"),
    (lambda: clip.grad_norm(HANDLE, [X]), "device"),
    (lambda: clip.grad_norm(HANDLE, [T]), "device|float32"),
    (lambda: clip.grad_norm(HANDLE, [3.0]), "tensors"),
    (lambda: clip.grad_norm(HANDLE, [X], max_norm=0.0), "positive"),
    (lambda: clip.grad_norm(HANDLE, [X], max_norm=float("nan")), "positive"),
    (lambda: clip.grad_norm(HANDLE, [X], max_norm=1.0, eps=-1.0), "negative"),
    (lambda: clip.grad_norm(HANDLE, [X], inv_scale=torch.ones(1)), "inv_scale"),
    (lambda: clip.clip_grads(HANDLE, [X], 1.0, out=[]), "each gradient"),
])
def test_the_binding_refuses(call, what):
    with pytest.raises(ValueError, match=what):
        call()


def test_the_library_refuses_without_a_handle(stq_lib):
    assert vocab._lib().stq_vocab_loss(None, None, 0, None, 0, None, None, -100, 0, 0, 0, None, None, None) == -1
    assert vocab._lib().stq_vocab_loss_backward(None, None, None, 0, None, 0, None, None, -100, None, 0, 0, 0, None, 0, None, 0, 0, None, None) == -1
    assert clip._lib().stq_grad_norm(None, None, 0, None, 1.0, 0.0, None, None, None, None) == -1
    assert clip._lib().stq_grad_clip(None, None, 0, None, 1.0, 0.0, None, None, None, None) == -1


def _dense(grads):
    try:
        return clip._lists.rows(grads, None, -1)[1] == 1
    except ValueError as e:
        assert "dense" in str(e)
        return False


def test_rows_of_a_list(stq_lib):
    """The layout of stq_grad, without the gradients that are None."""
    clip._lib()
    a, b = torch.zeros(3, 4, dtype=torch.bfloat16), torch.zeros(5)
    o = torch.zeros(3, 4), torch.zeros(5)
    import numpy as np
    rows, n = clip._lists.rows([a, None, b], [o[0], None, o[1]], -1)
    table = np.frombuffer(rows, dtype=np.uint64).reshape(2, 4)
    assert n == 2 and table[:, 0].tolist() == [a.data_ptr(), b.data_ptr()] and table[:, 1].tolist() == [o[0].data_ptr(), o[1].data_ptr()]
    assert table[:, 2].tolist() == [12, 5] and np.frombuffer(rows, dtype=np.int32).reshape(2, 8)[:, 6:].tolist() == [[1, 0], [0, 0]]
    for bad, what in ((([a], [torch.zeros(4, 3)]), "layout"), (([b], [torch.zeros(5, dtype=torch.bfloat16)]), "type of its gradient"),
                      (([b], []), "each gradient"), (([b], [None]), "results are tensors"), (([b.double()], None), "float64|Double")):
        with pytest.raises(ValueError, match=what):
            clip._lists.rows(*bad, -1)
    before = a._version, b._version
    clip._lists.written([a, None, b])
    assert (a._version, b._version) == (before[0] + 1, before[1] + 1)
    with torch.inference_mode():
        clip._lists.written([torch.zeros(3)])


def test_dense_layouts(stq_lib):
    clip._lib()
    x = torch.zeros(3, 4, 5)
    dense = lambda t: _dense([t])      # noqa: E731
    assert all(dense(t) for t in (x, x.transpose(0, 2), x.permute(1, 2, 0), x[:1].transpose(1, 2), torch.zeros(()), torch.zeros(0, 3)))
    assert not any(dense(t) for t in (x[:, :2], x[..., ::2], x[:1].expand(3, 4, 5), x[:, 0]))


def test_the_module_refuses():
    m = VocabLoss(64, 9, device="cpu")
    with pytest.raises(ValueError, match="bfloat16"):
        m(X.float(), T)
    with pytest.raises(ValueError, match="target"):
        m(X, T[:2])
    with pytest.raises(ValueError, match="reduction"):
        m(X, T, "max")
    with pytest.raises(ValueError, match="weight"):
        VocabLoss(64, 9, weight=torch.nn.Parameter(torch.zeros(9, 63)))
    tied = torch.nn.Parameter(torch.zeros(9, 64))
    assert VocabLoss(64, 9, weight=tied).weight is tied
