"""How far O of a row may be off whose keys are attended in two parts, shared and others, each with P in two bf16 operands.

Beyond accuracy_util.row_bound: the scale of V goes into the exponent of the shared part (scales within 2^-8 .. 2^8, their logarithm off by 2^-21, its difference
to the reference by 2^-21: 2^-20 of a probability), and the parts are joined, at most six steps one after the other, each with
an exponential and two products for a sum (2^-21) and a difference of references (2^-23 of the largest score): 2^-18 and 2^-20 of the largest score.  Numerator and
denominator are off by these."""
import torch

import accuracy_util as A


def bound(a, p, v, o):
    largest = torch.where(p > 0, a, 0.0).amax(1, keepdim=True)
    r = 2.0 ** -20 + 2.0 ** -18 + 2.0 ** -20 * largest
    return A.row_bound(a, p, v, o) + 1.01 * r * (p @ v.abs() + o.abs())


def model(p, v, shared, form):
    """O of probabilities p as a kernel makes it that holds those of the first `shared` keys, of the others, or none in one operand alone."""
    t = (p / p.amax(1, keepdim=True)).float().double()
    hi = A.bf16(t)
    lo = A.bf16(t - hi)
    if form == "shared":
        lo[:, :shared] = 0
    if form == "others":
        lo[:, shared:] = 0
    return A.bf16((hi + lo) @ v / t.sum(1, keepdim=True))
