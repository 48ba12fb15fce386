"""The bound of two bf16 operands of P, on the CPU: a model of the kernels' roundings keeps it, and with one operand, or a wrong second one,
does not, on rows of as few keys as those of tests/test_gpu_accuracy.py: that test would find such a kernel."""
import pytest
import torch

import accuracy_util as A


def cases():
    g = torch.Generator().manual_seed(0)
    for keys in (2, 3, 8, 40, 64):
        for d in (64, 128):
            q, k, v = (torch.randn(x, d, generator=g, dtype=torch.float64).to(torch.bfloat16).double() for x in (16, keys, keys))
            p = torch.softmax(q @ k.T * d ** -0.5, 1)
            yield q.abs() @ k.abs().T * d ** -0.5, p, v, p @ v


def test_two_operands_keep_the_bound():
    for a, p, v, o in cases():
        A.check(A.model(p, v, "two"), o, A.row_bound(a, p, v, o))


@pytest.mark.parametrize("form", ["one", "minus"])
def test_one_operand_and_a_wrong_second_one_do_not(form):
    for a, p, v, o in cases():
        with pytest.raises(AssertionError):
            A.check(A.model(p, v, form), o, A.row_bound(a, p, v, o))
