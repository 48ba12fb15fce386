"""The norm and turn of heads and their gradients by their definition in 64 bits (torch, on any device)."""
import numpy as np
import torch

F64 = torch.float64


def pairs(rot, interleaved):
    i = torch.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def turn(x, pos, freq, interleaved, factor=1.0, sign=1):
    """x [rows, heads, d] (float64) with its pairs turned by sign * pos * freq and multiplied by factor."""
    a, b = pairs(2 * len(freq), interleaved)
    angle = sign * pos.to(F64)[:, None, None] * torch.as_tensor(np.asarray(freq), device=x.device)
    c, s, y = factor * angle.cos(), factor * angle.sin(), x.clone()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def spread(x, freq, interleaved, factor=1.0):
    """|a| + |b| of each pair at both of its columns, |x| at the others: what the roundings of a turn are relative to."""
    a, b = pairs(2 * len(freq), interleaved)
    y = x.abs()
    y[..., a] = y[..., b] = factor * (x[..., a].abs() + x[..., b].abs())
    return y


def forward(x, pos, freq, interleaved, factor=1.0, gain=None, eps=1e-6):
    u = x.to(F64)
    if gain is not None:
        u = gain.to(F64) * u / (u.square().mean(-1, keepdim=True) + eps).sqrt()
    return turn(u, pos, freq, interleaved, factor), spread(u, freq, interleaved, factor)


def backward(x, dy, pos, freq, interleaved, factor=1.0, gain=None, eps=1e-6):
    """dx and dg, and what their roundings are relative to."""
    dy = dy.to(F64)
    u, far = turn(dy, pos, freq, interleaved, factor, -1), spread(dy, freq, interleaved, factor)
    if gain is None:
        return u, None, far, None
    x, g = x.to(F64), gain.to(F64)
    root = (x.square().mean(-1, keepdim=True) + eps).sqrt()
    xh = x / root
    dg, dg_far = (u * xh).sum((0, 1)), (far * xh.abs()).sum((0, 1))
    dx = (g * u - xh * (g * u * xh).mean(-1, keepdim=True)) / root
    return dx, dg, (g.abs() * far + xh.abs() * (g.abs() * far * xh.abs()).mean(-1, keepdim=True)) / root, dg_far


# Roundings.  fp32 (half a step: 2^-24 of a value): sine and cosine 2^-22 off (the series 2.5e-8, its roundings, the angle's), at most 20 additions of squares and a
# reciprocal root in the norm's factor, four products and sums behind: below 2^-19 of the pair's magnitudes together; of a gradient, with
# the mean of products in it, below 2^-18.  Then one rounding to bf16, 2^-8 of the value.
def close(got, want, far, fp32=2.0 ** -19):
    got = got.to(F64)
    off = (got - want).abs() - (2.0 ** -8 * want.abs() + fp32 * far + 1e-30)
    assert not torch.isnan(off).any() and off.max() <= 0, float(off.max())


# A gain's gradient: each term 2^-18 of its magnitudes, and sums of up to 512 terms one after the other (2^-15 of all magnitudes), at most 20 behind.
def close_gain(got, want, far):
    off = (got.to(F64) - want).abs() - (2.0 ** -15 + 2.0 ** -17) * far
    assert got.dtype == torch.float32 and not torch.isnan(off).any() and off.max() <= 0, float(off.max())
