"""The cache's definitions in 64 bits (numpy and torch on the CPU), and batches over a cache."""
import numpy as np
import torch

F8 = torch.float8_e4m3fn
PAGE = 64


def values(codes, scale):
    """What codes [pages, heads, x, y] stand for, as float64."""
    return codes.cpu().view(torch.uint8).view(F8).double() * scale.cpu().double()[:, :, None, None]


def round_e4m3(x):
    """float64 values of at most 448 to the nearest e4m3, ties to even: steps of 2^(e - 3) where 2^e <= |x|, of 2^-9 below 2^-6."""
    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -20))), -6.0) - 3)
    return np.rint(x / step) * step


def append(held, new, n, lens, table):
    """The cache after an append: held = {"k", "v" (values / scale, [page, head, token, dim]), "ks", "vs"} as float64 arrays, in
    place.  Sequences have n[i] new rows and lens[i] tokens with them."""
    row = 0
    for i, (r, total) in enumerate(zip(n, lens)):
        p = total - r
        while p < total:
            page, a = table[i, p // PAGE], p % PAGE
            e = min(PAGE, a + total - p)
            for x, codes, scale in ((new[0], held["k"][page], held["ks"][page]), (new[1], held["v"][page], held["vs"][page])):
                x = x[row:row + e - a].transpose(1, 0, 2)
                top = np.where(np.isfinite(x), np.abs(x), 0).max((1, 2))
                now = np.maximum(np.exp2(np.ceil(np.log2(np.maximum(top, 1e-300) / 448))), 2.0 ** -126)
                if a > 0:
                    now = np.maximum(now, scale)
                    codes[:] = round_e4m3(codes * (scale / now)[:, None, None])
                codes[:, a:e] = round_e4m3(x / now[:, None, None])
                scale[:] = now
            row, p = row + e - a, p + e - a


def attend(cache, q, n, lens, table, window=None, sinks=0, scale=None):
    """O and LSE (float64), and how far a kernel's O may be off that rounds P (relative to itself by at most 2^-8) and O to bf16."""
    k, v = values(cache.k, cache.k_scale), values(cache.v, cache.v_scale).transpose(2, 3)
    q = q.double().cpu()
    hq, d = q.shape[1:]
    g, scale = hq // k.shape[1], scale or d ** -0.5
    o, far, lse = torch.zeros_like(q), torch.zeros_like(q), torch.full((hq, q.shape[0]), -np.inf, dtype=torch.float64)
    row = 0
    for i, (r, total) in enumerate(zip(n, lens)):
        ids = torch.as_tensor(table[i, :-(-total // PAGE)]).long()
        there = ((ids >= 0) & (ids < k.shape[0])).repeat_interleave(PAGE)[:total]
        pos, j = torch.arange(total - r, total)[:, None], torch.arange(total)
        see = there & (j <= pos)
        if window is not None:
            see &= (pos - j < window) | (j < sinks)
        used = see.any(0)
        for h in range(hq):
            at = torch.where((ids >= 0) & (ids < k.shape[0]), ids, 0)
            kh, vh = (torch.where(used[:, None], x[at, h // g].reshape(-1, d)[:total], 0.0) for x in (k, v))
            s = (q[row:row + r, h] @ kh.T * scale).masked_fill(~see, -np.inf)
            part = torch.logsumexp(s, 1)
            p = torch.exp(s - torch.where(torch.isinf(part), 0.0, part)[:, None])
            o[row:row + r, h], far[row:row + r, h], lse[h, row:row + r] = p @ vh, p @ vh.abs(), part
        row += r
    return o, lse, 1.01 * 2.0 ** -8 * (far + o.abs()) + 1e-6


def check(got_o, got_lse, want, rows=None):
    o, lse, far = want
    rows = slice(None) if rows is None else rows
    x = got_o.double().cpu()[rows]
    assert torch.isfinite(x).all()
    off = (x - o[rows]).abs() - far[rows]
    assert off.max() <= 0, float(off.max())
    if got_lse is not None:
        y, z = got_lse.double().cpu()[:, rows], lse[:, rows]
        none = torch.isinf(z)
        assert (y[none] == -np.inf).all()
        assert ((y - z).abs()[~none] <= 1e-4 + 2.0 ** -20 * z.abs()[~none]).all()


def layout(lens, extra=3, seed=0):
    """A page table [sequences][pages], pages in no order, -1 behind a sequence's last; and how many pages there are."""
    need = [-(-x // PAGE) for x in lens]
    ids = np.random.default_rng(seed).permutation(sum(need) + extra)
    table, at = np.full((len(lens), max(need + [1])), -1, np.int32), 0
    for i, x in enumerate(need):
        table[i, :x] = ids[at:at + x]
        at += x
    return table, sum(need) + extra
