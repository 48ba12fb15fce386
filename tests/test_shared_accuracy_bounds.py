"""The bound of attention in two parts, on the CPU: with P in two operands it is kept, and with one for the shared keys, or for the others, it is not, on
rows as short as those of tests/test_gpu_shared_accuracy.py."""
import pytest
import torch

import accuracy_util as A
import shared_accuracy_util as S


def cases():
    g = torch.Generator().manual_seed(0)
    for shared, others in ((64, 40), (128, 130), (384, 300)):
        for d in (64, 128):
            q, k, v = (torch.randn(x, d, generator=g, dtype=torch.float64).to(torch.bfloat16).double() for x in (16, shared + others, shared + others))
            q = A.bf16(0.1 * q)
            p = torch.softmax(q @ k.T * d ** -0.5, 1)
            yield q.abs() @ k.abs().T * d ** -0.5, p, v, p @ v, shared


def test_two_operands_keep_the_bound():
    for a, p, v, o, shared in cases():
        A.check(S.model(p, v, shared, "two"), o, S.bound(a, p, v, o))


@pytest.mark.parametrize("form", ["shared", "others"])
def test_one_operand_for_either_part_does_not(form):
    for a, p, v, o, shared in cases():
        with pytest.raises(AssertionError):
            A.check(S.model(p, v, shared, form), o, S.bound(a, p, v, o))
