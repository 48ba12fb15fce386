"""Calls of the rotation with queries alone, or one side's tensors without the other's (no GPU)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2510_18121_amd import binding as B
from paper_2510_18121_amd import rotary as R

POS = torch.zeros(3, dtype=torch.int32)


def x(heads=2):
    return torch.zeros(3, heads, 64, dtype=torch.bfloat16)


@pytest.fixture
def calls(monkeypatch):
    """What reaches the library, which computes nothing; tensors on the CPU are taken for the device's."""
    made = []
    lib = SimpleNamespace(ca_rotate=lambda r, tensors, n, *rest: made.append(n) or 0, ca_rotate_backward=lambda r, tensors, n, *rest: made.append(n) or 0,
                          ca_rotate_backward_workspace_bytes=lambda: 1024)
    monkeypatch.setattr(B, "lib", lambda: lib)
    monkeypatch.setattr(B, "_rotate_stream", lambda rotation, stream: None)
    return made


@pytest.fixture
def rotation():
    r = R.Rotation(64, device="cpu")
    r.index = -1
    return r


def test_a_gain_or_an_output_of_no_keys(calls, rotation):
    gain = torch.ones(64)
    for kw in ({"k_gain": gain}, {"k_gain": gain, "q_gain": gain}):
        with pytest.raises(ValueError):
            rotation(x().requires_grad_(), None, POS, **kw)
        with pytest.raises(ValueError):
            B.ca_rotate(rotation, x(), None, x(), None, POS, **kw)
    with pytest.raises(ValueError):
        B.ca_rotate(rotation, x(), None, x(), x(), POS)
    assert calls == []
    rotation(x().requires_grad_(), None, POS, q_gain=gain)
    assert calls == [1]


def test_keys_without_an_output(calls, rotation):
    with pytest.raises(ValueError):
        B.ca_rotate(rotation, x(), x(1), x(), None, POS)
    with pytest.raises(ValueError):
        B.ca_rotate_backward(rotation, None, None, x(), x(1), x(), None, POS)
    assert calls == []


def test_gradients_that_nobody_would_write(calls, rotation):
    gain, ws = torch.ones(64), torch.zeros(1024, dtype=torch.uint8)
    for kw in ({"k_gain": gain, "dk_gain": torch.empty(64)}, {"dk_gain": torch.empty(64)}):
        with pytest.raises(ValueError):
            B.ca_rotate_backward(rotation, x(), None, x(), None, x(), None, POS, q_gain=gain, dq_gain=torch.empty(64), ws=ws, **kw)
    with pytest.raises(ValueError):
        B.ca_rotate_backward(rotation, None, None, x(), None, x(), x(), POS)
    with pytest.raises(ValueError):
        B.ca_rotate_backward(rotation, None, x(1), None, x(1), x(), x(1), POS)
    assert calls == []
    B.ca_rotate_backward(rotation, x(), None, x(), None, x(), None, POS, q_gain=gain, dq_gain=torch.empty(64), ws=ws)
    B.ca_rotate_backward(rotation, None, None, None, x(1), None, x(1), POS)
    assert calls == [1, 1]


def test_gradients_of_the_op_with_queries_alone(calls, rotation):
    q, gain = x().requires_grad_(), torch.ones(64, requires_grad=True)
    y = rotation(q, None, POS, q_gain=gain)
    dq, dg = torch.autograd.grad(y, (q, gain), torch.ones_like(y))
    assert dq.shape == q.shape and dg.shape == gain.shape and calls == [1, 1]
