"""Attention with a sliding window and sinks by its definition, in 64 bits on the CPU: a dense mask per document, for small batches."""
import numpy as np
import torch

from paper_2510_18121_amd import workloads as W


def batch(lens, tasks, hq, hkv, d, kv_lens=None, seed=0):
    """workloads.custom, with the keys of task i clipped to kv_lens[i] where that is given."""
    b = W.custom(lens, tasks, hq, hkv, d, seed=seed)
    for i, n in (kv_lens or {}).items():
        b.task_kv_len[i] = n
    return b


def visible(b, window, sinks):
    """bool [total_q, total_kv]: which packed keys each packed row sees (rows of no task: none)."""
    see = np.zeros((b.total_q, b.total_kv), bool)
    for t in range(b.n_tasks):
        doc, q0, n, p0, kv = (int(x[t]) for x in (b.task_doc, b.task_q_start, b.task_q_len, b.task_q_pos, b.task_kv_len))
        p, j = np.arange(p0, p0 + n)[:, None], np.arange(int(b.doc_kv_len[doc]))[None]
        k0 = int(b.doc_kv_start[doc])
        see[q0:q0 + n, k0:k0 + j.shape[1]] = (j < kv) & (j <= p) & ((p - j < window) | (j < sinks))
    return see


def reference(b, window, sinks, q, k, v, d_o=None, o_given=None):
    """O, LSE and, with d_o, dQ, dK, dV in float64 (the tensors are on any device and of any type); o_given: the O of <dO, O>.  And
    for each result but LSE how far a kernel may be off that rounds P and dS (relative to themselves by at most half a step of bf16, 2^-8)
    before the products with them, sums in fp32, and rounds the result to bf16: 2^-8 (sum of the products' magnitudes + the
    result's magnitude), 1 % more for second order, and 2^-15 of the magnitudes that cancel in dP - Delta for fp32 sums and
    exponentials (each relative 2^-24 times at most 2^9 terms)."""
    see = torch.from_numpy(visible(b, window, sinks))
    g, half = b.n_q_heads // b.n_kv_heads, 2.0 ** -8
    q, k, v = (x.detach().double().cpu() for x in (q, k, v))
    out = {n: torch.zeros_like(x) for n, x in (("o", q), ("dq", q), ("dk", k), ("dv", v))}
    far = {n: torch.zeros_like(x) for n, x in out.items()}
    out["lse"] = torch.full((b.n_q_heads, b.total_q), -np.inf, dtype=torch.float64)
    for h in range(b.n_q_heads):
        kh, vh = k[:, h // g], v[:, h // g]
        s = (q[:, h] @ kh.T * b.scale).masked_fill(~see, -np.inf)
        lse = torch.logsumexp(s, 1)
        p = torch.exp(s - torch.where(torch.isinf(lse), 0.0, lse)[:, None])
        out["lse"][h], out["o"][:, h], far["o"][:, h] = lse, p @ vh, half * (p @ vh.abs())
        if d_o is not None:
            do = d_o[:, h].double().cpu()
            o = out["o"][:, h] if o_given is None else o_given[:, h].double().cpu()
            ds = p * (do @ vh.T - (do * o).sum(1, keepdim=True))
            off = half * ds.abs() + 2.0 ** -15 * p * (do.abs() @ vh.abs().T + (do * o).abs().sum(1, keepdim=True))
            out["dq"][:, h], far["dq"][:, h] = ds @ kh * b.scale, off @ kh.abs() * b.scale
            out["dk"][:, h // g] += ds.T @ q[:, h] * b.scale
            far["dk"][:, h // g] += off.T @ q[:, h].abs() * b.scale
            out["dv"][:, h // g] += p.T @ do
            far["dv"][:, h // g] += half * (p.T @ do.abs())
    return out, {n: 1.01 * (x + half * out[n].abs()) + 1e-6 for n, x in far.items()}


def check(got, want, far, names):
    for n in names:
        x = got[n].double().cpu()
        assert torch.isfinite(x).all(), n
        off = (x - want[n]).abs() - far[n]
        assert off.max() <= 0, (n, float(off.max()), int(off.argmax()))
