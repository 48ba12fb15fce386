"""Attention with a sliding window and sinks, and a cache of keys and values in 8 bits: the operators as measurable cases.

kind "window": core attention over the CA-tasks of a batch where a row at document position p sees, of the keys
j < min(kv_len, p + 1), those with p - j < window or j < sinks.  Forward, forward + backward ("step"), and the differentiable
op ("train").
kind "attend": queries of sequences (single tokens, or chunks of a prompt) over a paged cache of e4m3 codes with one scale per
(page of 64 tokens, KV head), with or without a window.
kind "append": new tokens of sequences quantised into their pages; a page's scale is the smallest power of two that holds its
tokens, and what a page holds (its 64 tokens) is rounded again where its scale grows.
kind "copy": pages copied within a cache, as a fork of sequences or a compaction of the pool needs.

Sequence s has the rows q_start[s] .. q_start[s + 1] - 1, which sit at its positions kv_len[s] - rows .. kv_len[s] - 1.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

DEV = "cuda:0"
PAGE = 64
F8 = torch.float8_e4m3fn
BLOCK = 128  # rows that the plain form of the windowed attention takes together


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # the smallest server call: a document and a bit in two shards, a small head layout (inference of a short prompt)
        {"name": "window_tiny_fwd", "kind": "window", "run": "fwd", "tokens": 385, "median": 300, "shard": 200, "window": 128, "sinks": 4,
         "hq": 4, "hkv": 2, "d": 64, "layout": 31},
        # a training micro-batch of packed documents, multi-head, head_dim 64, through the differentiable op
        {"name": "window_mha_d64_16k_train", "kind": "window", "run": "train", "tokens": 16411, "median": 2048, "shard": 0, "window": 512,
         "sinks": 0, "hq": 16, "hkv": 16, "d": 64, "layout": 32},
        # a 64K-token chunk of long documents in shuffled shards, 8B-class heads, with sinks: forward and backward
        {"name": "window_64k_step", "kind": "window", "run": "step", "tokens": 65536, "median": 24576, "shard": 4096, "window": 1024, "sinks": 4,
         "hq": 32, "hkv": 8, "d": 128, "layout": 33},
        # one token of one sequence: where latency counts
        {"name": "cache_decode_1x901", "kind": "attend", "seqs": 1, "rows": 1, "median": 901, "spread": 0.0, "window": 0, "sinks": 0, "hq": 32,
         "hkv": 8, "d": 128, "layout": 34},
        # a decoding batch of unlike lengths
        {"name": "cache_decode_64_ragged", "kind": "attend", "seqs": 64, "rows": 1, "median": 4096, "spread": 1.0, "window": 0, "sinks": 0,
         "hq": 32, "hkv": 8, "d": 128, "layout": 35},
        # a few sequences with 128K of context, 70B-class heads
        {"name": "cache_decode_4x128k", "kind": "attend", "seqs": 4, "rows": 1, "median": 130001, "spread": 0.0, "window": 0, "sinks": 0,
         "hq": 64, "hkv": 8, "d": 128, "layout": 36},
        # decoding with a sliding window and sinks, head_dim 64
        {"name": "cache_decode_32_window", "kind": "attend", "seqs": 32, "rows": 1, "median": 16000, "spread": 0.7, "window": 4096, "sinks": 4,
         "hq": 16, "hkv": 16, "d": 64, "layout": 37},
        # chunks of prompts behind what the cache holds of them
        {"name": "cache_chunk_4x500", "kind": "attend", "seqs": 4, "rows": 500, "median": 8192, "spread": 0.3, "window": 0, "sinks": 0,
         "hq": 32, "hkv": 8, "d": 128, "layout": 38},
        # one token of each sequence of a decoding batch into the cache
        {"name": "cache_append_128x1", "kind": "append", "seqs": 128, "rows": 1, "median": 1024, "spread": 0.8, "hkv": 8, "d": 128, "layout": 39},
        # prompts of unlike lengths into the cache, half of them behind tokens that are there already
        {"name": "cache_append_16x2k", "kind": "append", "seqs": 16, "rows": 2048, "median": 3000, "spread": 0.5, "hkv": 8, "d": 128,
         "layout": 40},
        # sixteen sequences forked inside a page: their last pages are copied
        {"name": "cache_copy_16", "kind": "copy", "pages": 64, "pairs": 16, "hkv": 8, "d": 128, "layout": 41},
        # a pool compacted
        {"name": "cache_copy_4000", "kind": "copy", "pages": 10007, "pairs": 4000, "hkv": 8, "d": 128, "layout": 42},
    ]


HEADS = ((4, 2), (8, 1), (8, 2), (6, 2), (16, 16), (32, 8), (64, 8))


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(("window", "window", "window", "attend", "attend", "attend", "append", "copy"))
        hq, hkv = rng.choice(HEADS)
        c = {"kind": kind, "hq": hq, "hkv": hkv, "d": rng.choice((64, 128, 128)), "layout": rng.randrange(1 << 20)}
        if kind == "window":
            c |= {"run": rng.choice(("fwd", "step", "train")), "tokens": _log(rng, 200, 65536), "median": _log(rng, 64, 32768),
                  "shard": rng.choice((0, _log(rng, 16, 8192))), "window": _log(rng, 1, 8192), "sinks": rng.choice((0, 0, 1, 4, 16, 130))}
            b = _tasks(c)
            blocks = int(((b.task_q_len + BLOCK - 1) // BLOCK).sum())
            if blocks * BLOCK * hq * (c["window"] + c["sinks"] + BLOCK) * 4 > 10.5e9 or _window_pairs(c) * hq * c["d"] > 2.8e11:
                continue
        elif kind == "attend":
            rows = rng.choice((1, 1, 1, _log(rng, 2, 600)))
            c |= {"seqs": _log(rng, 1, 200 if rows == 1 else 8), "rows": rows, "median": _log(rng, 16, 130000), "spread": rng.choice((0.0, 0.5, 1.0)),
                  "window": rng.choice((0, 0, _log(rng, 16, 8192))), "sinks": rng.choice((0, 4, 70))}
            n, lens = _lengths(c)
            if len(n) * max(lens) * hkv * c["d"] * 4 > 9.5e9 or len(n) * max(n) * hq * max(lens) * 4 > 9.5e9:
                continue
        elif kind == "append":
            rows = rng.choice((1, _log(rng, 2, 4000)))
            c |= {"seqs": _log(rng, 1, 256 if rows == 1 else 16), "rows": rows, "median": _log(rng, 16, 6000), "spread": rng.choice((0.0, 0.5, 1.0))}
            del c["hq"]
            if sum(_lengths(c)[1]) * hkv * c["d"] > 2e8:
                continue
        else:
            pages = _log(rng, 8, 10000)
            c |= {"pages": pages, "pairs": _log(rng, 1, pages // 2)}
            del c["hq"]
        return c


# ------------------------------------------------------------------------------------------------ what the cases consist of
def _tasks(c):
    """The batch of CA-tasks of a windowed case: ragged documents, cut into shards of `shard` rows (0: not cut), shards shuffled."""
    rng = random.Random(c["layout"])
    lens, left = [], c["tokens"]
    while left > 0:
        lens.append(min(left, max(1, round(rng.lognormvariate(math.log(c["median"]), 1.0)))))
        left -= lens[-1]
    tasks = [(i, a, min(c["shard"] or n, n - a)) for i, n in enumerate(lens) for a in range(0, n, c["shard"] or n)]
    rng.shuffle(tasks)
    doc, pos, n = (np.array(x, np.int64) for x in zip(*tasks))
    start = np.cumsum(lens) - np.array(lens)
    return SimpleNamespace(n_q_heads=c["hq"], n_kv_heads=c["hkv"], head_dim=c["d"], total_q=int(n.sum()), total_kv=sum(lens), softmax_scale=0.0,
                           doc_kv_start=start, doc_kv_len=np.array(lens, np.int64), task_doc=doc, task_q_start=np.cumsum(n) - n, task_q_len=n,
                           task_q_pos=pos, task_kv_len=pos + n)


def _window_pairs(c):
    """(row, key) pairs that are seen: of a document of n keys, sum over p of min(p + 1, window) + the sinks before the window."""
    total = 0
    for n in _tasks(c).doc_kv_len.tolist():
        w, k = min(c["window"], n), min(c["sinks"], n)
        total += w * (w + 1) // 2 + (n - w) * w
        far = n - w  # rows p >= w: min(sinks, p + 1 - w) further keys
        total += far * (far + 1) // 2 if far <= k else k * (k + 1) // 2 + (far - k) * k
    return total


def _lengths(c):
    """(rows, keys) of each sequence of a cache case; a chunk's rows are `rows` and fewer, and sit at the end of the keys."""
    rng = random.Random(c["layout"])
    n, lens = [], []
    for _ in range(c["seqs"]):
        total = max(1, round(rng.lognormvariate(math.log(c["median"]), c["spread"])))
        r = c["rows"] if c["rows"] == 1 else rng.randint(c["rows"] // 2 + 1, c["rows"])
        if c["kind"] == "append" and rng.random() < 0.5 and c["rows"] > 1:
            total = r  # a prompt from its first token
        n.append(r)
        lens.append(max(total, r))
    return n, lens


def _seen(n, total, window, sinks):
    """Keys of `total` that some of the last n rows sees, and (row, key) pairs."""
    if not window or window >= total:
        return total, n * (2 * total - n + 1) // 2
    first = max(0, total - n - window + 1)
    pairs = 0
    for p in (range(total - n, total)):
        pairs += min(p + 1, window) + min(sinks, max(0, p + 1 - window))
    return total - first + min(sinks, first), pairs


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(gen, *shape):
    out = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 26):  # in pieces, so that the fp32 staging stays small
        m = min(1 << 26, flat.numel() - i)
        flat[i:i + m] = torch.randn(m, generator=gen, device=DEV)
    return out


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _filled(gen, pages, hkv, d, power_of_two):
    """A pool of pages as it is in use: codes of N(0, 1) at the scale of each (page, head), keys of some pages larger than of others."""
    k = torch.empty(pages, hkv, PAGE, d, dtype=F8, device=DEV)
    v = torch.empty(pages, hkv, d, PAGE, dtype=F8, device=DEV)
    ks, vs = (torch.empty(pages, hkv, device=DEV) for _ in range(2))
    for a in range(0, pages, 2048):
        for codes, scale in ((k, ks), (v, vs)):
            x = torch.randn(codes[a:a + 2048].shape, generator=gen, device=DEV)
            x *= torch.rand(x.shape[:2], generator=gen, device=DEV)[:, :, None, None] * 0.5 + 0.75
            s = x.abs().amax((2, 3)) / 448
            if power_of_two:
                s = torch.exp2(torch.ceil(torch.log2(s)))
            scale[a:a + 2048] = s
            codes[a:a + 2048] = (x / s[:, :, None, None]).clamp(-448, 448).to(F8)
    return k, v, ks, vs


def _tables(c, lens):
    """Pages of each sequence, in no order; -1 behind its last one.  Eight pages belong to nobody."""
    need = [-(-x // PAGE) for x in lens]
    ids = list(range(sum(need) + 8))
    random.Random(c["layout"] + 1).shuffle(ids)
    table = np.full((len(lens), max(need)), -1, np.int32)
    for s, x in enumerate(need):
        table[s, :x] = ids[:x]
        del ids[:x]
    return table, sum(need) + 8


def prepare(c, seed):
    g = _gen(seed)
    s = {"case": c}
    if c["kind"] == "window":
        b = _tasks(c)
        s["q"], s["k"], s["v"], s["do"] = (_normal(g, n, h, c["d"]) for n, h in ((b.total_q, c["hq"]), (b.total_kv, c["hkv"]), (b.total_kv, c["hkv"]),
                                                                                (b.total_q, c["hq"])))
        s["blocks"] = int(((b.task_q_len + BLOCK - 1) // BLOCK).sum())
        s["tasks"] = {n: torch.tensor(getattr(b, "task_" + n), device=DEV) for n in ("q_start", "q_len", "q_pos", "kv_len")}
        s["tasks"]["kv_start"] = torch.tensor(b.doc_kv_start[b.task_doc], device=DEV)
        if own:  # the plan and its workspace
            from paper_2510_18121_amd import binding as B
            from paper_2510_18121_amd.autograd import AttentionServer
            if c["run"] == "train":
                s["server"] = AttentionServer(b, DEV, window=c["window"], sinks=c["sinks"])
                for n in ("q", "k", "v"):
                    s[n].requires_grad_()
            else:
                s["plan"] = B.ca_plan(b, window=c["window"], sinks=c["sinks"])
                s["ws"] = B.alloc_workspace(s["plan"], DEV)
            s["o"], s["lse"] = torch.empty_like(s["q"]), torch.empty(c["hq"], b.total_q, device=DEV)
            s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[n]) for n in ("q", "k", "v"))
        return s
    if c["kind"] == "copy":
        ids = list(range(c["pages"]))
        random.Random(c["layout"]).shuffle(ids)
        s["k"], s["v"], s["ks"], s["vs"] = _filled(g, c["pages"], c["hkv"], c["d"], True)
        s["src"], s["dst"] = _i32(ids[:c["pairs"]]), _i32(ids[c["pairs"]:2 * c["pairs"]])
    else:
        n, lens = _lengths(c)
        table, pages = _tables(c, lens)
        s["rows"], s["keys"] = max(n), max(lens)
        s["q_start"], s["kv_len"], s["table"] = _i32([0] + np.cumsum(n).tolist()), _i32(lens), torch.tensor(table, device=DEV)
        s["k"], s["v"], s["ks"], s["vs"] = _filled(g, pages, c["hkv"], c["d"], c["kind"] == "append")
        if c["kind"] == "append":
            s["new_k"], s["new_v"] = (_normal(g, sum(n), c["hkv"], c["d"]) for _ in range(2))
        else:
            s["q"] = _normal(g, sum(n), c["hq"], c["d"])
            s["o"], s["lse"] = torch.empty_like(s["q"]), torch.empty(c["hq"], sum(n), device=DEV)
    if own:
        from paper_2510_18121_amd import binding as B
        from paper_2510_18121_amd.cache import KVCache
        s["cache"] = KVCache(s["k"], s["v"], s["ks"], s["vs"])
        if c["kind"] == "attend":
            s["ws"] = B.alloc_cache_workspace(s["cache"], c["hq"], DEV)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    c = s["case"]
    if c["kind"] == "window":
        return _run_window(s, c) if own else _plain_window(s, c)
    if c["kind"] == "attend":
        return _run_attend(s, c) if own else _plain_attend(s, c)
    if c["kind"] == "append":
        if own:
            from paper_2510_18121_amd import binding as B
            B.ca_cache_append(s["cache"], s["new_k"], s["new_v"], s["q_start"], s["kv_len"], s["table"])
        else:
            _plain_append(s)
    elif own:
        from paper_2510_18121_amd import binding as B
        B.ca_cache_copy_pages(s["cache"], s["src"], s["dst"])
    else:
        src, dst = s["src"].long(), s["dst"].long()
        for x in (s["k"].view(torch.uint8), s["v"].view(torch.uint8), s["ks"], s["vs"]):
            x[dst] = x[src]
    return {"k": s["k"], "v": s["v"], "k_scale": s["ks"], "v_scale": s["vs"]}


def _run_window(s, c):
    from paper_2510_18121_amd import binding as B
    if c["run"] == "train":
        o = s["server"](s["q"], s["k"], s["v"])
        dq, dk, dv = torch.autograd.grad(o, (s["q"], s["k"], s["v"]), s["do"])
        return {"o": o, "dq": dq, "dk": dk, "dv": dv}
    B.ca_forward(s["plan"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["ws"])
    if c["run"] == "fwd":
        return {"o": s["o"], "lse": s["lse"]}
    B.ca_backward(s["plan"], s["q"], s["k"], s["v"], s["o"], s["do"], s["lse"], s["dq"], s["dk"], s["dv"], s["ws"])
    return {n: s[n] for n in ("o", "lse", "dq", "dk", "dv")}


def _run_attend(s, c):
    from paper_2510_18121_amd import binding as B
    B.ca_cache_attend(s["cache"], s["q"], s["o"], s["lse"], s["q_start"], s["kv_len"], s["table"], s["ws"], window=c["window"] or None,
                      sinks=c["sinks"])
    return {"o": s["o"], "lse": s["lse"]}


def _softmax(x):
    """Probabilities and log-sum-exp over the last axis; rows of -inf alone get 0 and -inf."""
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = (x - m).exp_()
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total == 0, 1.0, total), (m + total.log()).squeeze(-1)


def _plain_window(s, c):
    """BLOCK rows of a task at a time against the sinks and the window + BLOCK - 1 keys that one of them may see, all blocks at once in fp32."""
    t, hkv, d, w, sinks = s["tasks"], c["hkv"], c["d"], c["window"], c["sinks"]
    g, total_q = c["hq"] // hkv, s["q"].shape[0]
    ends = ((t["q_len"] + BLOCK - 1) // BLOCK).cumsum(0)
    block = torch.arange(s["blocks"], device=DEV)
    task = torch.searchsorted(ends, block, right=True)
    t = {n: x[task][:, None] for n, x in t.items()}
    at = (block[:, None] - (ends[task][:, None] - (t["q_len"] + BLOCK - 1) // BLOCK)) * BLOCK
    i = at + torch.arange(BLOCK, device=DEV)
    row, pos = torch.where(i < t["q_len"], t["q_start"] + i, total_q), t["q_pos"] + i  # rows behind a task's last one: a row that is dropped
    band = t["q_pos"] + at - (w - 1) + torch.arange(w + BLOCK - 1, device=DEV)
    key = torch.cat([torch.arange(sinks, device=DEV).expand(s["blocks"], -1), torch.where(band < sinks, -1, band)], 1)
    key_ok = (key >= 0) & (key < t["kv_len"])
    seen = key_ok[:, None] & (key[:, None] <= pos[:, :, None]) & ((pos[:, :, None] - key[:, None] < w) | (key[:, None] < sinks))
    seen = (seen & (i < t["q_len"])[:, :, None])[:, None, None]
    at_kv = t["kv_start"] + torch.where(key_ok, key, 0)
    rows_of = lambda x: x.detach()[row.clamp(max=total_q - 1)].float().view(-1, BLOCK, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(-1, hkv, g * BLOCK, d)  # noqa: E731
    q, k, v = rows_of(s["q"]), s["k"].detach()[at_kv].float().transpose(1, 2), s["v"].detach()[at_kv].float().transpose(1, 2)
    scores = (q @ k.transpose(2, 3)).mul_(1 / math.sqrt(d)).view(-1, hkv, g, BLOCK, key.shape[1])
    p, lse = _softmax(scores.masked_fill_(~seen, -math.inf))
    del scores
    p = p.view(-1, hkv, g * BLOCK, key.shape[1])
    o = p @ v

    def back(x):
        out = torch.empty(total_q + 1, c["hq"], d, dtype=torch.bfloat16, device=DEV)
        out[row] = x.view(-1, hkv, g, BLOCK, d).permute(0, 3, 1, 2, 4).reshape(-1, BLOCK, c["hq"], d).to(torch.bfloat16)
        return out[:total_q]

    out = {"o": back(o)}
    if c["run"] != "train":
        lse_rows = torch.empty(total_q + 1, c["hq"], device=DEV)
        lse_rows[row] = lse.permute(0, 3, 1, 2).reshape(-1, BLOCK, c["hq"])
        out["lse"] = lse_rows[:total_q].t().contiguous()
    if c["run"] == "fwd":
        return out
    do = rows_of(s["do"])
    ds = (do @ v.transpose(2, 3)).sub_((do * o).sum(-1, keepdim=True)).mul_(p)
    sums = lambda x: torch.zeros(s["k"].shape, device=DEV).index_add_(0, at_kv.reshape(-1), x.transpose(1, 2).reshape(-1, hkv, d)).to(torch.bfloat16)  # noqa: E731
    out["dv"] = sums(p.transpose(2, 3) @ do)
    del p
    out["dq"] = back((ds @ k).mul_(1 / math.sqrt(d)))
    out["dk"] = sums((ds.transpose(2, 3) @ q).mul_(1 / math.sqrt(d)))
    return out


def _plain_attend(s, c):
    hkv, d, g = c["hkv"], c["d"], c["hq"] // c["hkv"]
    total_q = s["q"].shape[0]
    start, kv_len, table = s["q_start"].long(), s["kv_len"].long()[:, None], s["table"].long().clamp(min=0)
    k = (s["k"].view(torch.uint8)[table].view(F8).float() * s["ks"][table][..., None, None]).permute(0, 2, 1, 3, 4).reshape(-1, hkv, table.shape[1] * PAGE, d)
    v = (s["v"].view(torch.uint8)[table].view(F8).float() * s["vs"][table][..., None, None]).permute(0, 2, 1, 4, 3).reshape(-1, hkv, table.shape[1] * PAGE, d)
    i = torch.arange(s["rows"], device=DEV)[None]
    n = (start[1:] - start[:-1])[:, None]
    row, pos = torch.where(i < n, start[:-1, None] + i, total_q), kv_len - n + i
    q = s["q"][row.clamp(max=total_q - 1)].float().view(-1, s["rows"], hkv, g, d).permute(0, 2, 3, 1, 4).reshape(-1, hkv, g * s["rows"], d)
    key = torch.arange(k.shape[2], device=DEV)
    seen = (key < kv_len)[:, None] & (key <= pos[:, :, None])
    if c["window"]:
        seen &= (pos[:, :, None] - key < c["window"]) | (key < c["sinks"])
    x = (q @ k.transpose(2, 3)).mul_(1 / math.sqrt(d)).view(-1, hkv, g, s["rows"], key.numel()).masked_fill_(~seen[:, None, None], -math.inf)
    p, lse = _softmax(x)
    o = (p.view(-1, hkv, g * s["rows"], key.numel()) @ v).view(-1, hkv, g, s["rows"], d).permute(0, 3, 1, 2, 4)
    out, out_lse = torch.empty(total_q + 1, c["hq"], d, dtype=torch.bfloat16, device=DEV), torch.empty(total_q + 1, c["hq"], device=DEV)
    out[row] = o.reshape(-1, s["rows"], c["hq"], d).to(torch.bfloat16)
    out_lse[row] = lse.permute(0, 3, 1, 2).reshape(-1, s["rows"], c["hq"])
    return {"o": out[:total_q], "lse": out_lse[:total_q].t().contiguous()}


def _plain_append(s):
    start, kv_len, table = s["q_start"].long(), s["kv_len"].long(), s["table"].long()
    first = kv_len - (start[1:] - start[:-1])  # the position of each sequence's first new token
    token = torch.arange(s["new_k"].shape[0], device=DEV)
    seq = torch.searchsorted(start, token, right=True) - 1
    pos = first[seq] + token - start[seq]
    page, slot = table[seq, pos // PAGE], pos % PAGE
    partial = table[torch.arange(len(kv_len), device=DEV), first // PAGE]  # the pages that may hold tokens already
    fresh = (first % PAGE == 0)[:, None]
    for new, codes, scale, by_token in ((s["new_k"], s["k"], s["ks"], True), (s["new_v"], s["v"], s["vs"], False)):
        top = torch.zeros_like(scale).scatter_reduce_(0, page[:, None].expand(-1, scale.shape[1]), new.float().abs().amax(2), "amax")
        m, e = torch.frexp(top)  # the smallest power of two that is at least top / 448 (448 = 0.875 * 2^9)
        need = torch.ldexp(torch.ones_like(top), torch.where(m > 0.875, e - 8, e - 9).clamp(min=-126))
        old = scale[partial]
        now = torch.where(fresh, need[partial], torch.maximum(old, need[partial]))
        held = codes.view(torch.uint8)[partial].view(F8).float() * torch.where(fresh, 1.0, old / now)[..., None, None]
        codes.view(torch.uint8)[partial] = held.to(F8).view(torch.uint8)
        scale[page] = need[page]
        scale[partial] = now
        x = (new.float() / scale[page][:, :, None]).to(F8).view(torch.uint8)
        if by_token:
            codes.view(torch.uint8)[page, :, slot] = x
        else:
            codes.view(torch.uint8)[page, :, :, slot] = x


# ------------------------------------------------------------------------------------------------ what is asked of them
def work(c):
    if c["kind"] == "window":  # forward: Q, K, V in, O and LSE out; with backward also dO in, dQ, dK, dV out
        b = _tasks(c)
        qb, kb, lb = 2 * b.total_q * c["hq"] * c["d"], 2 * b.total_kv * c["hkv"] * c["d"], 4 * c["hq"] * b.total_q
        return {"bytes": 2 * qb + 2 * kb + lb if c["run"] == "fwd" else 4 * qb + 4 * kb + lb,
                "flops": (4 if c["run"] == "fwd" else 14) * c["d"] * c["hq"] * _window_pairs(c)}
    if c["kind"] == "copy":
        return {"bytes": 2 * c["pairs"] * c["hkv"] * (2 * PAGE * c["d"] + 8), "flops": 0}
    n, lens = _lengths(c)
    if c["kind"] == "append":  # bf16 K and V in, codes out, scales in and out
        pages = sum(-(-x // PAGE) - (x - r) // PAGE for r, x in zip(n, lens))
        return {"bytes": sum(n) * c["hkv"] * c["d"] * 6 + pages * c["hkv"] * 16, "flops": 4 * sum(n) * c["hkv"] * c["d"]}
    seen = [_seen(r, x, c["window"], c["sinks"]) for r, x in zip(n, lens)]
    keys, pairs = sum(x[0] for x in seen), sum(x[1] for x in seen)
    return {"bytes": keys * c["hkv"] * 2 * c["d"] + keys // PAGE * c["hkv"] * 8 + sum(n) * c["hq"] * (4 * c["d"] + 4), "flops": 4 * pairs * c["hq"] * c["d"]}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(c, seed):
    return {"window": _exact_window, "attend": _exact_attend, "append": _exact_append, "copy": _exact_copy}[c["kind"]](c, prepare(c, seed))


def _exact_window(c, s):
    """Task by task, a run of rows against all the keys up to the last one that a row of it sees."""
    b, f64, hkv, d, w, sinks = _tasks(c), torch.float64, c["hkv"], c["d"], c["window"], c["sinks"]
    g = c["hq"] // hkv
    q, k, v, do = (s[n].detach() for n in ("q", "k", "v", "do"))
    out = {"o": torch.zeros(q.shape, dtype=f64, device=DEV), "lse": torch.zeros(c["hq"], b.total_q, dtype=f64, device=DEV)}
    out |= {"dq": torch.zeros_like(out["o"]), "dk": torch.zeros(k.shape, dtype=f64, device=DEV), "dv": torch.zeros(k.shape, dtype=f64, device=DEV)}
    for doc, q0, n, p0 in zip(b.task_doc.tolist(), b.task_q_start.tolist(), b.task_q_len.tolist(), b.task_q_pos.tolist()):
        kv0 = int(b.doc_kv_start[doc])
        step = max(64, min(2048, w))
        for a in range(0, n, step):
            e = min(n, a + step)
            pos = torch.arange(p0 + a, p0 + e, device=DEV)[:, None]
            keys = torch.arange(p0 + e, device=DEV)
            keys = keys[(keys < sinks) | (keys > p0 + a - w)]
            hidden = (keys > pos) | ((pos - keys >= w) & (keys >= sinks))
            at, rows = kv0 + keys, slice(q0 + a, q0 + e)
            kt, vt = k[at].to(f64).transpose(0, 1), v[at].to(f64).transpose(0, 1)
            qt = q[rows].to(f64).transpose(0, 1).reshape(hkv, g * (e - a), d)
            x = torch.bmm(qt, kt.transpose(1, 2).contiguous()).div_(math.sqrt(d)).view(hkv, g, e - a, -1).masked_fill_(hidden, -math.inf).view(hkv, g * (e - a), -1)
            lse = torch.logsumexp(x, 2, keepdim=True)
            x.sub_(lse).exp_()
            ot = torch.bmm(x, vt)
            out["o"][rows] = ot.view(c["hq"], e - a, d).transpose(0, 1)
            out["lse"][:, rows] = lse.view(c["hq"], e - a)
            if c["run"] == "fwd":
                continue
            dt = do[rows].to(f64).transpose(0, 1).reshape(hkv, g * (e - a), d)
            out["dv"].index_add_(0, at, torch.bmm(x.transpose(1, 2).contiguous(), dt).transpose(0, 1))
            ds = torch.bmm(dt, vt.transpose(1, 2).contiguous()).sub_((dt * ot).sum(2, keepdim=True)).mul_(x).div_(math.sqrt(d))
            out["dq"][rows] = torch.bmm(ds, kt).view(c["hq"], e - a, d).transpose(0, 1)
            out["dk"].index_add_(0, at, torch.bmm(ds.transpose(1, 2).contiguous(), qt).transpose(0, 1))
    return {n: out[n] for n in {"fwd": ("o", "lse"), "step": ("o", "lse", "dq", "dk", "dv"), "train": ("o", "dq", "dk", "dv")}[c["run"]]}


def _exact_attend(c, s):
    f64, hkv, d = torch.float64, c["hkv"], c["d"]
    g = c["hq"] // hkv
    o, lse = torch.zeros(s["q"].shape, dtype=f64, device=DEV), torch.zeros(c["hq"], s["q"].shape[0], dtype=f64, device=DEV)
    row = 0
    for i, (n, total) in enumerate(zip(*_lengths(c))):
        pages = s["table"][i, :-(-total // PAGE)].long()
        pos = torch.arange(total - n, total, device=DEV)[:, None]
        key = torch.arange(total, device=DEV)
        hidden = key > pos
        if c["window"]:
            hidden |= (key <= pos - c["window"]) & (key >= c["sinks"])
        for h in range(hkv):
            kt = (s["k"][:, h].view(torch.uint8)[pages].view(F8).to(f64) * s["ks"][pages, h].to(f64)[:, None, None]).reshape(-1, d)[:total]
            vt = (s["v"][:, h].view(torch.uint8)[pages].view(F8).to(f64) * s["vs"][pages, h].to(f64)[:, None, None]).transpose(1, 2).reshape(-1, d)[:total]
            qt = s["q"][row:row + n, h * g:(h + 1) * g].to(f64).transpose(0, 1)
            x = ((qt.reshape(g * n, d) @ kt.t().contiguous()) / math.sqrt(d)).view(g, n, total).masked_fill_(hidden, -math.inf)
            total_lse = torch.logsumexp(x, 2)
            o[row:row + n, h * g:(h + 1) * g] = ((x - total_lse[:, :, None]).exp_().view(g * n, total) @ vt).view(g, n, d).transpose(0, 1)
            lse[h * g:(h + 1) * g, row:row + n] = total_lse
        row += n
    return {"o": o, "lse": lse}


def _to_e4m3(x):
    """The nearest e4m3 value, ties to even, of float64 values of at most 448: steps of 2^(e - 3) for 2^e <= |x|, of 2^-9 below 2^-6."""
    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -20))), -6.0) - 3)
    return np.rint(x / step) * step


def _exact_append(c, s):
    host = {n: s[n].double().cpu().numpy() for n in ("k", "v", "ks", "vs", "new_k", "new_v")}
    table = s["table"].cpu().numpy()
    row = 0
    for i, (n, total) in enumerate(zip(*_lengths(c))):
        p = total - n
        while p < total:  # a page at a time
            page, a = table[i, p // PAGE], p % PAGE
            e = min(PAGE, a + total - p)
            for new, codes, scale in (("new_k", host["k"][page], host["ks"][page]), ("new_v", host["v"][page].transpose(0, 2, 1), host["vs"][page])):
                x = host[new][row:row + e - a].transpose(1, 0, 2)
                need = np.maximum(np.exp2(np.ceil(np.log2(np.maximum(np.abs(x).max((1, 2)), 1e-300) / 448))), 2.0 ** -126)
                now = need if a == 0 else np.maximum(need, scale)
                if a > 0:  # (all of it: what lies behind the new tokens is nobody's, but it is there)
                    codes[:] = _to_e4m3(codes * (scale / now)[:, None, None])
                codes[:, a:e] = _to_e4m3(x / now[:, None, None])
                scale[:] = now
            row, p = row + e - a, p + e - a
    return {"k": torch.from_numpy(host["k"]), "v": torch.from_numpy(host["v"]), "k_scale": torch.from_numpy(host["ks"]),
            "v_scale": torch.from_numpy(host["vs"])}


def _exact_copy(c, s):
    src, dst = s["src"].tolist(), s["dst"].tolist()
    out = {}
    for name, key in (("k", "k"), ("v", "v"), ("k_scale", "ks"), ("v_scale", "vs")):
        x = s[key].view(torch.uint8) if s[key].dtype == F8 else s[key]
        kept = x.clone()
        for a in range(0, len(src), 512):
            kept.index_copy_(0, torch.tensor(dst[a:a + 512], device=DEV), x.index_select(0, torch.tensor(src[a:a + 512], device=DEV)))
        out[name] = kept.view(F8) if s[key].dtype == F8 else kept.double()
    return out
