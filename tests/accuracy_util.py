"""Softmax rows whose probabilities are held in two bf16 operands (hi + lo): their O in 64 bits and how far a kernel's may be off, and a model
of such a kernel's roundings on the CPU.

The bound, from the roundings alone.  A score is an fp32 sum of D exact products (bf16 times bf16 or e4m3): off by at most D 2^-24 a with
a = scale sum |q k|, and with the factors of the exponent (three roundings, counted as 8) by (D + 8) 2^-24 a; the difference to the row's reference adds
2^-24 of at most twice the largest a, the exponential 2^-22 of its result.  So a probability is off by r = (D + 8) 2^-24 a + 2^-23 max a + 2^-22 of
itself.  hi + lo leaves 2^-8 2^-8 of it, scales and fp32 sums of n terms (n + 4) 2^-24.  O's numerator and denominator are off by these, and O's own
rounding by 2^-8 of O; 1 % more for second order."""
import numpy as np
import torch


def row_bound(a, p, v, o):
    """a: [rows, keys] scale sum |q k|, p: probabilities, v: [keys, dim], o = p v, all float64; keys that are not seen have p = 0."""
    d, n = v.shape[1], (p > 0).sum(1, keepdim=True).double()
    a = torch.where(p > 0, a, 0.0)
    r = (d + 8) * 2.0 ** -24 * a + 2.0 ** -23 * a.amax(1, keepdim=True) + 2.0 ** -22
    sums = (n + 4) * 2.0 ** -24
    off = (p * (r + 2.0 ** -16 + sums)) @ v.abs() + o.abs() * ((p * r).sum(1, keepdim=True) + sums)
    return 1.01 * (off + 2.0 ** -8 * o.abs()) + 1e-30


def bf16(x):
    return x.float().to(torch.bfloat16).double()


def model(p, v, form):
    """O of rows of probabilities p (float64), as a kernel makes it: relative to the largest, held in two bf16 operands ("two"), in one ("one"), or in
    two whose second is wrong ("minus")."""
    t = (p / p.amax(1, keepdim=True).clamp(min=1e-300)).float().double()
    hi = bf16(t)
    lo = bf16(t - hi)
    held = {"two": hi + lo, "one": hi, "minus": hi - lo}[form]
    total = t.sum(1, keepdim=True)
    return bf16(torch.where(total > 0, held @ v / torch.where(total > 0, total, 1.0), 0.0))


def check(got, o, bound):
    x = got.double().cpu()
    assert torch.isfinite(x).all()
    off = (x - o).abs() - bound
    assert off.max() <= 0, (float(off.max()), int(off.argmax()))


def cache_rows(values_k, values_v, q, n, lens, table, window, sinks):
    """Of a call on a cache, for each sequence and query head: rows, a, p, v and O (see row_bound).  values_*: [pages, heads, token, dim]."""
    hq, d = q.shape[1:]
    g, row = hq // values_k.shape[1], 0
    for i, (r, total) in enumerate(zip(n, lens)):
        ids = torch.as_tensor(np.asarray(table[i, :-(-total // 64)])).long()
        pos, j = torch.arange(total - r, total)[:, None], torch.arange(total)
        see = (j <= pos) if window is None else (j <= pos) & ((pos - j < window) | (j < sinks))
        for h in range(hq):
            k, v = (x[ids, h // g].reshape(-1, d)[:total] for x in (values_k, values_v))
            qh = q[row:row + r, h].double().cpu()
            s = (qh @ k.T * d ** -0.5).masked_fill(~see, -np.inf)
            p = torch.softmax(s, 1)
            yield slice(row, row + r), h, qh.abs() @ k.abs().T * d ** -0.5, p, v, p @ v
        row += r
