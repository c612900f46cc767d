"""The 8-bit operators refuse what they cannot take before anything reaches a device (no GPU)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2604_06836_b200 import q8

HANDLE = SimpleNamespace(device=0, _h=None)      # (no call below gets as far as using it)
X, W = torch.zeros(4, 64), torch.ones(64)
ROWS = q8.Rows8(torch.zeros(4, 64, dtype=torch.int8), torch.ones(4))


@pytest.mark.parametrize("call,what", [
    (lambda: q8.norm(HANDLE, X, W), "device"),
    (lambda: q8.norm(HANDLE, X[0], W), "matrix"),
    (lambda: q8.norm(HANDLE, X.half(), W), "float32 or bfloat16"),
    (lambda: q8.quantize_rows(HANDLE, X.to(torch.int32)), "float32 or bfloat16"),
    (lambda: q8.norm_backward(HANDLE, X, X, W, torch.ones(4)), "device"),
    (lambda: q8.act(HANDLE, X, "tanh"), "kind"),
    (lambda: q8.act(HANDLE, X, "gelu"), "device"),
    (lambda: q8.act_backward(HANDLE, X, q8.Checkpoint8(torch.zeros(4, 1, 64, dtype=torch.int8), torch.ones(4, 1, 1), 64, "silu_gated")),
     "parts"),
    (lambda: q8.act_backward(HANDLE, X, q8.Checkpoint8(torch.zeros(4, 1, 64, dtype=torch.int8), torch.ones(4, 2, 1), 64, "gelu")),
     "act"),
    (lambda: q8.linear(HANDLE, ROWS, ROWS), "device"),
    (lambda: q8.linear(HANDLE, ROWS, ROWS, dtype=torch.float16), "float32 or bfloat16"),
    (lambda: q8.linear_dx(HANDLE, X, ROWS), "device"),
    (lambda: q8.linear_dw(HANDLE, X, ROWS), "device"),
    (lambda: q8.bias_grad(HANDLE, X), "device"),
])
def test_the_binding_refuses(call, what):
    with pytest.raises(ValueError, match=what):
        call()


def test_the_library_refuses_without_a_handle(stq_lib):
    L = q8._lib()
    assert L.stq_q8_rows(None, None, 0, 0, 0, 0, None, 0, None, None) == -1
    assert L.stq_q8_norm(None, None, 0, None, 0, None, 1.0, 0, 0, 0, None, 0, None, None, 0, None, None, 0, None) == -1
    assert L.stq_q8_norm_backward(None, None, 0, None, 0, None, None, None, 0, 0, 0, 0, None, 0, None, None) == -1
    assert L.stq_q8_act(None, None, 0, 0, 0, 0, 0, None, 0, None, None, 0, None, 0, None, None) == -1
    assert L.stq_q8_act_backward(None, None, 0, 0, 0, 0, 0, None, 0, None, None, 0, None) == -1
    assert L.stq_q8_linear(None, None, 0, None, None, 0, None, None, 0, 0, 0, None, 0, 0, None) == -1
    assert L.stq_q8_linear_dx(None, None, 0, None, 0, None, 0, 0, 0, None, 0, 0, None) == -1
    assert L.stq_q8_linear_dw(None, None, 0, None, 0, None, 0, 0, 0, None, 0, 0, None) == -1
    assert L.stq_q8_bias_grad(None, None, 0, 0, 0, 0, None, None) == -1


def test_rows_and_checkpoints_decode_on_the_host():
    r = q8.Rows8(torch.tensor([[-127, 0, 127]], dtype=torch.int8), torch.tensor([0.5]))
    assert r.values().tolist() == [[-63.5, 0.0, 63.5]]
    q = torch.zeros(1, 2, 144, dtype=torch.int8)
    q[0, 0, 127], q[0, 0, 128], q[0, 1, 129] = 1, 2, 3
    c = q8.Checkpoint8(q, torch.tensor([[[1.0, 10.0], [100.0, 1000.0]]]), 130, "silu_gated")
    v = c.values()
    assert v.shape == (1, 260) and v[0, 127] == 1 and v[0, 128] == 20 and v[0, 130 + 129] == 3000 and int((v != 0).sum()) == 3
    assert c.nbytes() == 288 + 16
    a = q8.alloc_rows(3, 17, "cpu")
    assert a.q.shape == (3, 17) and a.q.stride() == (32, 1) and a.scale.shape == (3,)
