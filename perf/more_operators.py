"""Queries and keys turned by their positions, a cache in 8 bits read back, and attention of sequences that share a prefix: the operators as
measurable cases.

kind "rotate": queries and keys of packed rows, each (row, head) divided by its root mean square and multiplied by a gain (or not), its
first `rot` columns turned by the row's position: pairs (i, i + rot / 2), or (2 i, 2 i + 1) where interleaved.  Out of a joint tensor of
queries, keys and values ("fwd"), for new tokens of cached sequences ("serve"), and the differentiable op with its gradients ("train").
kind "read": tokens of sequences back out of a paged cache of e4m3 codes, one scale per (page of 64 tokens, KV head).
kind "shared": queries of sequences over such a cache, where groups of sequences have their first pages in common.

Sequence s has the rows q_start[s] .. q_start[s + 1] - 1, which sit at its positions kv_len[s] - rows .. kv_len[s] - 1.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
PAGE = 64
F8 = torch.float8_e4m3fn
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # one new token of one sequence, between its projections and the cache: where latency counts
        {"name": "rotate_serve_1", "kind": "rotate", "run": "serve", "rows": 1, "hq": 32, "hkv": 8, "d": 128, "rot": 128, "interleaved": False,
         "norm": True, "far": 8, "layout": 51},
        # a decoding batch with long contexts, 70B-class heads, turned but not normed
        {"name": "rotate_serve_250", "kind": "rotate", "run": "serve", "rows": 250, "hq": 64, "hkv": 8, "d": 128, "rot": 128, "interleaved": False,
         "norm": False, "far": 8, "layout": 52},
        # a prompt far into a long context, out of the joint projection
        {"name": "rotate_fwd_40001", "kind": "rotate", "run": "fwd", "rows": 40001, "hq": 32, "hkv": 8, "d": 128, "rot": 128, "interleaved": True,
         "norm": False, "far": 8, "layout": 53},
        # a training micro-batch, multi-head, head_dim 64, half of each head turned
        {"name": "rotate_train_16k_d64", "kind": "rotate", "run": "train", "rows": 16411, "hq": 16, "hkv": 16, "d": 64, "rot": 32, "interleaved": True,
         "norm": True, "far": 1, "layout": 54},
        # a 64K-token chunk of packed documents, 8B-class heads, gains of both norms learnt
        {"name": "rotate_train_64k", "kind": "rotate", "run": "train", "rows": 65536, "hq": 32, "hkv": 8, "d": 128, "rot": 128, "interleaved": False,
         "norm": True, "far": 4, "layout": 55},
        # the last tokens of a few sequences
        {"name": "read_3x40", "kind": "read", "seqs": 3, "rows": 40, "median": 700, "spread": 0.5, "hkv": 8, "d": 128, "layout": 56},
        # whole contexts, as a prefill in 16 bits or a move to another server reads them
        {"name": "read_8x16k", "kind": "read", "seqs": 8, "rows": 0, "median": 16000, "spread": 0.7, "hkv": 8, "d": 128, "layout": 57},
        # a handful of answers to one prompt
        {"name": "shared_8x2k", "kind": "shared", "groups": 1, "seqs": 8, "rows": 1, "prefix": 2048, "uneven": 0.0, "median": 90, "spread": 0.6,
         "hq": 32, "hkv": 8, "d": 128, "layout": 58},
        # a decoding batch behind one long system prompt
        {"name": "shared_64x8k", "kind": "shared", "groups": 1, "seqs": 64, "rows": 1, "prefix": 8192, "uneven": 0.0, "median": 500, "spread": 0.8,
         "hq": 32, "hkv": 8, "d": 128, "layout": 59},
        # questions about several documents at a time, multi-head, head_dim 64
        {"name": "shared_200_of_9_d64", "kind": "shared", "groups": 9, "seqs": 200, "rows": 1, "prefix": 4000, "uneven": 0.8, "median": 300,
         "spread": 0.8, "hq": 16, "hkv": 16, "d": 64, "layout": 60},
        # drafts of several tokens each, checked together
        {"name": "shared_24x5_rows", "kind": "shared", "groups": 2, "seqs": 24, "rows": 5, "prefix": 6000, "uneven": 0.3, "median": 700, "spread": 0.5,
         "hq": 32, "hkv": 8, "d": 128, "layout": 61},
        # many answers over a context of 128K tokens, 70B-class heads
        {"name": "shared_32x128k", "kind": "shared", "groups": 1, "seqs": 32, "rows": 1, "prefix": 130048, "uneven": 0.0, "median": 1500,
         "spread": 0.6, "hq": 64, "hkv": 8, "d": 128, "layout": 62},
    ]


HEADS = ((4, 2), (8, 1), (8, 2), (6, 2), (16, 16), (32, 8), (64, 8))


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(("rotate", "rotate", "read", "shared", "shared", "shared"))
        hq, hkv = rng.choice(HEADS)
        c = {"kind": kind, "hq": hq, "hkv": hkv, "d": rng.choice((64, 128, 128)), "layout": rng.randrange(1 << 20)}
        if kind == "rotate":
            run = rng.choice(("serve", "fwd", "train", "train"))
            c |= {"run": run, "rows": _log(rng, 1, 400 if run == "serve" else 65536),
                  "rot": rng.choice((c["d"], c["d"], c["d"] // 2, c["d"] // 4, 2 * rng.randint(1, c["d"] // 2))), "interleaved": rng.random() < 0.4,
                  "norm": rng.random() < 0.6, "far": rng.choice((1, 4, 8))}
            if c["rows"] * (hq + hkv) * c["d"] > 65536 * 40 * 128:
                continue
        elif kind == "read":
            c |= {"seqs": _log(rng, 1, 100), "rows": rng.choice((0, 0, _log(rng, 1, 2000))), "median": _log(rng, 16, 60000),
                  "spread": rng.choice((0.0, 0.5, 1.0))}
            del c["hq"]
            if sum(_lengths(c)[0]) * hkv * c["d"] > 1.5e8:
                continue
        else:
            seqs = _log(rng, 2, 256)
            c |= {"seqs": seqs, "groups": rng.choice((1, 1, _log(rng, 1, seqs // 2))), "rows": rng.choice((1, 1, rng.randint(2, 9))),
                  "prefix": _log(rng, 40, 130000), "uneven": rng.choice((0.0, 0.6, 1.2)), "median": _log(rng, 4, 6000),
                  "spread": rng.choice((0.0, 0.5, 1.0))}
            members, prefix, n, tails = _groups(c)
            if seqs * (max(tails) + PAGE) * hkv * c["d"] * 4 > 8e9 or seqs * max(n) * hq * (max(tails) + PAGE) * 4 > 8e9:
                continue
            if max(m * max(n) * p for m, p in zip(members, prefix)) * hq * 4 > 4e9 or sum(prefix) * hkv * c["d"] > 6e8:
                continue
            if _pairs(c) * hq * c["d"] > 32 * 131000 * 64 * 128:
                continue
        return c


# ------------------------------------------------------------------------------------------------ what the cases consist of
def _positions(c):
    """Packed documents whose rows begin anywhere in their contexts; `far` 1, 4, 8: contexts up to 32K, 128K, a million."""
    rng = random.Random(c["layout"])
    top, out = {1: 1 << 15, 4: 1 << 17, 8: 1 << 20}[c["far"]], []
    while len(out) < c["rows"]:
        n = min(c["rows"] - len(out), max(1, round(rng.lognormvariate(math.log(2500), 1.2))))
        first = rng.choice((0, rng.randrange(top)))
        out += range(first, first + n)
    return np.array(out, np.int64)


def _served(c):
    """(rows, tokens) of each sequence of a serving call: single tokens, and a few of several rows."""
    rng = random.Random(c["layout"])
    n, lens = [], []
    while sum(n) < c["rows"]:
        n.append(min(c["rows"] - sum(n), rng.choice((1, 1, 1, 1, rng.randint(2, 5)))))
        lens.append(n[-1] + _log(rng, 1, {1: 1 << 15, 4: 1 << 17, 8: 1 << 20}[c["far"]]))
    return n, lens


def _frequencies(c):
    """Radians per position of each pair.  For long contexts (`far` above 1) those that turn less than once in 8192 positions are slowed
    down by `far`, those that turn more than 32 times are not, and the ones between partly."""
    f = 500000.0 ** (-2 * np.arange(c["rot"] // 2) / c["rot"])
    if c["far"] == 1:
        return f
    kept = np.clip((8192 * f / (2 * math.pi) - 1) / 31, 0, 1)
    return f * (kept + (1 - kept) / c["far"])


def _magnitude(c):
    """The factor of cosines and sines that goes with the slowed frequencies."""
    return 1 + 0.1 * math.log(c["far"])


def _lengths(c):
    """(rows, tokens) of each sequence of a cache that is read; rows 0: all of them."""
    rng = random.Random(c["layout"])
    n, lens = [], []
    for _ in range(c["seqs"]):
        lens.append(max(1, round(rng.lognormvariate(math.log(c["median"]), c["spread"]))))
        n.append(min(lens[-1], rng.randint(c["rows"] // 2 + 1, c["rows"])) if c["rows"] else lens[-1])
    return n, lens


def _groups(c):
    """Sequences and prefix tokens (whole pages) of each group; rows, and tokens behind the prefix (the rows among them), of each sequence."""
    rng = random.Random(c["layout"])
    members = [2] * c["groups"]
    for _ in range(c["seqs"] - sum(members)):
        members[rng.randrange(c["groups"])] += 1
    prefix = [max(PAGE, round(c["prefix"] * math.exp(c["uneven"] * rng.uniform(-1, 0)) / PAGE) * PAGE) for _ in members]
    n = [rng.randint(c["rows"] // 2 + 1, c["rows"]) for _ in range(c["seqs"])]
    return members, prefix, n, [max(r, round(rng.lognormvariate(math.log(c["median"]), c["spread"]))) for r in n]


def _pairs(c):
    """(row, key) pairs that are seen."""
    members, prefix, n, tails = _groups(c)
    before = np.repeat(prefix, members).tolist()
    return sum(r * p + r * (2 * x - r + 1) // 2 for p, r, x in zip(before, n, tails))


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
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _start(n):
    return _i32([0] + np.cumsum(n).tolist())


def _filled(gen, pages, hkv, d):
    """A pool of pages as it is in use: codes of N(0, 1) at the scale of each (page, head), some pages larger than others."""
    k = torch.empty(pages, hkv, PAGE, d, dtype=F8, device=DEV)
    v = torch.empty(pages, hkv, d, PAGE, dtype=F8, device=DEV)
    ks, vs = (torch.empty(pages, hkv, device=DEV) for _ in range(2))
    for a in range(0, pages, 2048):
        for codes, scale in ((k, ks), (v, vs)):
            x = torch.randn(codes[a:a + 2048].shape, generator=gen, device=DEV)
            x *= torch.rand(x.shape[:2], generator=gen, device=DEV)[:, :, None, None] * 0.5 + 0.75
            s = x.abs().amax((2, 3)) / 448
            scale[a:a + 2048] = s
            codes[a:a + 2048] = (x / s[:, :, None, None]).clamp(-448, 448).to(F8)
    return k, v, ks, vs


def _tables(c, first, lens):
    """Pages of each sequence, in no order, -1 behind its last one; of those that go together (`first`: members and prefix pages) the first
    are the same.  Eight pages belong to nobody."""
    need = [-(-x // PAGE) for x in lens]
    pages = sum(need) - sum((m - 1) * p for m, p in first) + 8
    ids = list(range(pages))
    random.Random(c["layout"] + 1).shuffle(ids)
    table, s = np.full((len(lens), max(need)), -1, np.int32), 0
    for m, p in first:
        table[s:s + m, :p] = ids[:p]
        del ids[:p]
        for i in range(s, s + m):
            own_pages = need[i] - p
            table[i, p:need[i]] = ids[:own_pages]
            del ids[:own_pages]
        s += m
    return table, pages


def prepare(c, seed):
    g = _gen(seed)
    s = {"case": c}
    if c["kind"] == "rotate":
        hq, hkv, d, rows = c["hq"], c["hkv"], c["d"], c["rows"]
        if c["run"] == "train":
            s["q"], s["k"], s["dyq"], s["dyk"] = (_normal(g, rows, h, d) for h in (hq, hkv, hq, hkv))
            s["pos"] = _i32(_positions(c))
        else:
            joint = _normal(g, rows, (hq + 2 * hkv) * d)  # queries, keys and values side by side, as one projection gives them
            s["q"], s["k"] = joint[:, :hq * d].unflatten(1, (hq, d)), joint[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
            s["yq"], s["yk"] = (torch.empty(rows, h, d, dtype=torch.bfloat16, device=DEV) for h in (hq, hkv))
            if c["run"] == "serve":
                n, lens = _served(c)
                s["q_start"], s["kv_len"] = _start(n), _i32(lens)
            else:
                s["pos"] = _i32(_positions(c))
        s["gq"], s["gk"] = (1 + 0.2 * torch.randn(d, generator=g, device=DEV) for _ in range(2)) if c["norm"] else (None, None)
        s["freq"] = torch.tensor(_frequencies(c), device=DEV)
        if own:
            from paper_2510_18121_amd.rotary import Rotation
            s["rotation"] = Rotation(d, frequencies=_frequencies(c), interleaved=c["interleaved"], factor=_magnitude(c), device=DEV)
            if c["run"] == "train":
                s["leaves"] = [s[x].requires_grad_() for x in (("q", "k", "gq", "gk") if c["norm"] else ("q", "k"))]
        return s
    if c["kind"] == "read":
        n, lens = _lengths(c)
        first = [(1, 0)] * len(lens)
    else:
        members, prefix, n, tails = _groups(c)
        first, lens = [(m, p // PAGE) for m, p in zip(members, prefix)], (np.repeat(prefix, members) + tails).tolist()
    table, pages = _tables(c, first, lens)
    s["k"], s["v"], s["ks"], s["vs"] = _filled(g, pages, c["hkv"], c["d"])
    s["q_start"], s["kv_len"], s["table"] = _start(n), _i32(lens), torch.tensor(table, device=DEV)
    if c["kind"] == "read":
        s["k_out"], s["v_out"] = (torch.empty(sum(n), c["hkv"], c["d"], dtype=torch.bfloat16, device=DEV) for _ in range(2))
    else:
        s["q"] = _normal(g, sum(n), c["hq"], c["d"])
        s["o"], s["lse"] = torch.empty_like(s["q"]), torch.empty(c["hq"], sum(n), device=DEV)
        s["group_start"], s["prefix_pages"] = _start(members), _i32([p for _, p in first])
        s["members"], s["pages"], s["rows"], s["longest"] = members, [p for _, p in first], n, max(tails)
    if own:
        from paper_2510_18121_amd import binding as B
        from paper_2510_18121_amd.cache import KVCache
        s["cache"] = KVCache(s["k"], s["v"], s["ks"], s["vs"])
        if c["kind"] == "shared":
            s["ws"] = B.alloc_shared_workspace(s["cache"], c["hq"], sum(n))
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    c = s["case"]
    if c["kind"] == "rotate":
        return _run_rotate(s, c) if own else _plain_rotate(s, c)
    if c["kind"] == "shared":
        return _run_shared(s) if own else _plain_shared(s, c)
    if own:
        from paper_2510_18121_amd import binding as B
        B.ca_cache_read(s["cache"], s["k_out"], s["v_out"], s["q_start"], s["kv_len"], s["table"])
        return {"k": s["k_out"], "v": s["v_out"]}
    return _plain_read(s)


def _run_rotate(s, c):
    if c["run"] == "train":
        yq, yk = s["rotation"](s["q"], s["k"], s["pos"], q_gain=s["gq"], k_gain=s["gk"], eps=EPS)
        grads = torch.autograd.grad((yq, yk), s["leaves"], (s["dyq"], s["dyk"]))
        return {"q": yq.detach(), "k": yk.detach()} | dict(zip(("dq", "dk", "dgq", "dgk"), grads))
    from paper_2510_18121_amd import binding as B
    where = (s["q_start"], s["kv_len"]) if c["run"] == "serve" else None
    B.ca_rotate(s["rotation"], s["q"], s["k"], s["yq"], s["yk"], s.get("pos"), where=where, q_gain=s["gq"], k_gain=s["gk"], eps=EPS)
    return {"q": s["yq"], "k": s["yk"]}


def _run_shared(s):
    from paper_2510_18121_amd import binding as B
    B.ca_cache_attend_shared(s["cache"], s["q"], s["o"], s["lse"], s["q_start"], s["kv_len"], s["table"], s["group_start"], s["prefix_pages"], s["ws"])
    return {"o": s["o"], "lse": s["lse"]}


def _turned(x, cos, sin, rot, interleaved):
    """x [rows, heads, d] with its pairs turned by the angles of cos and sin [rows, rot / 2]."""
    cos, sin = cos[:, None], sin[:, None]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    a, b = a * cos - b * sin, a * sin + b * cos
    pairs = torch.stack((a, b), -1).flatten(2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((pairs, x[..., rot:]), -1) if rot < x.shape[-1] else pairs


def _plain_rotate(s, c):
    if c["run"] == "serve":
        start, token = s["q_start"].long(), torch.arange(c["rows"], device=DEV)
        seq = torch.searchsorted(start, token, right=True) - 1
        pos = s["kv_len"].long()[seq] + token - start[seq + 1]
    else:
        pos = s["pos"]
    angle = pos.double()[:, None] * s["freq"]  # in 64 bits: a million positions
    cos, sin = (f(angle).mul_(_magnitude(c)).float() for f in (torch.cos, torch.sin))
    out = {}
    for x in ("q", "k"):
        y = s[x].float()
        if c["norm"]:
            r = torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
            unit = y * r
            y = unit * s["g" + x]
        out[x] = _turned(y, cos, sin, c["rot"], c["interleaved"]).to(torch.bfloat16)
        if c["run"] != "train":
            continue
        u = _turned(s["dy" + x].float(), cos, -sin, c["rot"], c["interleaved"])
        if c["norm"]:
            out["dg" + x] = (u * unit).sum((0, 1), dtype=torch.float64).float()
            u = u * s["g" + x]
            u = r * (u - unit * (u * unit).mean(-1, keepdim=True))
        out["d" + x] = u.to(torch.bfloat16)
    return out


def _plain_read(s):
    start, token = s["q_start"].long(), torch.arange(s["k_out"].shape[0], device=DEV)
    seq = torch.searchsorted(start, token, right=True) - 1
    pos = s["kv_len"].long()[seq] + token - start[seq + 1]
    page, slot = s["table"].long()[seq, pos // PAGE], pos % PAGE
    return {"k": (s["k"].view(torch.uint8)[page, :, slot].view(F8).float() * s["ks"][page][:, :, None]).to(torch.bfloat16),
            "v": (s["v"].view(torch.uint8)[page, :, :, slot].view(F8).float() * s["vs"][page][:, :, None]).to(torch.bfloat16)}


def _softmax(x):
    """Probabilities and log-sum-exp over the last axis, of which every row sees some key."""
    m = x.amax(-1, keepdim=True)
    e = x.sub_(m).exp_()
    total = e.sum(-1, keepdim=True)
    return e.div_(total), (m + total.log()).squeeze(-1)


def _values(s, pages):
    """K and V [.., heads, tokens, d] of page ids [.., n], in fp32."""
    k = s["k"].view(torch.uint8)[pages].view(F8).float() * s["ks"][pages][..., None, None]
    v = (s["v"].view(torch.uint8)[pages].view(F8).float() * s["vs"][pages][..., None, None]).transpose(-1, -2)
    return (x.transpose(-4, -3).flatten(-3, -2) for x in (k, v))


def _plain_shared(s, c):
    """The prefix of each group once, against all rows of the group; then what is behind it, padded to the longest; joined by the log-sum-exps."""
    hkv, d, g = c["hkv"], c["d"], c["hq"] // c["hkv"]
    table = s["table"].long().clamp(min=0)
    q = s["q"].float().mul_(1 / math.sqrt(d))
    o, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    row = seq = 0
    for m, p in zip(s["members"], s["pages"]):
        rows = sum(s["rows"][seq:seq + m])
        k, v = _values(s, table[seq, :p])
        x = q[row:row + rows].view(rows, hkv, g, d).transpose(0, 1).reshape(hkv, rows * g, d)
        prob, part = _softmax(x @ k.transpose(1, 2))
        o[row:row + rows] = (prob @ v).view(hkv, rows, g, d).transpose(0, 1).reshape(rows, c["hq"], d)
        lse[row:row + rows] = part.view(hkv, rows, g).transpose(0, 1).reshape(rows, c["hq"])
        row, seq = row + rows, seq + m
    start, lens = s["q_start"].long(), s["kv_len"].long()
    behind = torch.repeat_interleave(s["prefix_pages"].long(), (s["group_start"][1:] - s["group_start"][:-1]).long(), output_size=len(s["rows"]))
    at = behind[:, None] + torch.arange(-(-s["longest"] // PAGE), device=DEV)
    k, v = _values(s, table.gather(1, at.clamp(max=table.shape[1] - 1)))
    n, i = start[1:] - start[:-1], torch.arange(max(s["rows"]), device=DEV)
    index = torch.where(i < n[:, None], start[:-1, None] + i, q.shape[0])  # (rows that a sequence does not have: one that is dropped)
    pos = (lens - n)[:, None] + i - behind[:, None] * PAGE
    hidden = torch.arange(k.shape[2], device=DEV) > pos[:, :, None]
    x = q[index.clamp(max=q.shape[0] - 1)].view(-1, i.numel(), hkv, g, d).permute(0, 2, 3, 1, 4).reshape(-1, hkv, g * i.numel(), d)
    x = (x @ k.transpose(2, 3)).view(-1, hkv, g, i.numel(), k.shape[2]).masked_fill_(hidden[:, None, None], -math.inf)
    prob, part = _softmax(x)
    own_o = (prob.view(-1, hkv, g * i.numel(), k.shape[2]) @ v).view(-1, hkv, g, i.numel(), d).permute(0, 3, 1, 2, 4).reshape(-1, i.numel(), c["hq"], d)
    o2, lse2 = torch.empty(q.shape[0] + 1, c["hq"], d, device=DEV), torch.empty(q.shape[0] + 1, c["hq"], device=DEV)
    o2[index], lse2[index] = own_o, part.permute(0, 3, 1, 2).reshape(-1, i.numel(), c["hq"])
    o2, lse2 = o2[:-1], lse2[:-1]
    top = torch.maximum(lse, lse2)
    a, b = (lse - top).exp_(), (lse2 - top).exp_()
    total = a + b
    return {"o": (o * (a / total)[..., None] + o2 * (b / total)[..., None]).to(torch.bfloat16), "lse": (top + total.log()).t().contiguous()}


# ------------------------------------------------------------------------------------------------ what is asked of them
def work(c):
    if c["kind"] == "rotate":  # queries and keys in and out; with gradients also those of the outputs in, those of the inputs out
        elements = c["rows"] * (c["hq"] + c["hkv"]) * c["d"]
        return {"bytes": (8 if c["run"] == "train" else 4) * elements + 4 * c["rows"], "flops": (20 if c["run"] == "train" else 7) * elements}
    if c["kind"] == "read":  # codes of K and V in, bf16 out
        n, _ = _lengths(c)
        return {"bytes": sum(n) * c["hkv"] * c["d"] * 6, "flops": 2 * sum(n) * c["hkv"] * c["d"]}
    _, prefix, n, tails = _groups(c)
    tokens = sum(prefix) + sum(tails)
    return {"bytes": tokens * c["hkv"] * 2 * c["d"] + tokens // PAGE * c["hkv"] * 8 + sum(n) * c["hq"] * (4 * c["d"] + 4),
            "flops": 4 * _pairs(c) * c["hq"] * c["d"]}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(c, seed):
    return {"rotate": _exact_rotate, "read": _exact_read, "shared": _exact_shared}[c["kind"]](c, prepare(c, seed))


def _exact_rotate(c, s):
    """Each pair as a complex number; a run of rows at a time."""
    f64, rot, d = torch.float64, c["rot"], c["d"]
    if c["run"] == "serve":
        pos = torch.tensor(np.concatenate([np.arange(x - r, x) for r, x in zip(*_served(c))]), device=DEV)
    else:
        pos = torch.tensor(_positions(c), device=DEV)
    even = torch.arange(0, rot, 2, device=DEV) if c["interleaved"] else torch.arange(rot // 2, device=DEV)
    odd = even + (1 if c["interleaved"] else rot // 2)
    out = {}
    for x in ("q", "k"):
        values, grads = s[x].detach(), s.get("dy" + x)
        y = torch.empty(values.shape, dtype=f64, device=DEV)
        dx, dg = torch.empty_like(y) if grads is not None else None, torch.zeros(d, dtype=f64, device=DEV)
        gain = s["g" + x].detach().to(f64) if c["norm"] else None
        for a in range(0, c["rows"], 8192):
            rows = slice(a, a + 8192)
            angle = pos[rows].to(f64)[:, None] * torch.tensor(_frequencies(c), device=DEV)
            turn = torch.polar(torch.full_like(angle, _magnitude(c)), angle)[:, None]
            z = values[rows].to(f64)
            if c["norm"]:
                root = (z.pow(2).sum(2, keepdim=True) / d + EPS).sqrt()
                z = z / root
            w = z * gain if c["norm"] else z.clone()
            pairs = torch.complex(w[..., even], w[..., odd]) * turn
            w[..., even], w[..., odd] = pairs.real, pairs.imag
            y[rows] = w
            if grads is None:
                continue
            u = grads[rows].to(f64)
            pairs = torch.complex(u[..., even], u[..., odd]) * turn.conj()
            u[..., even], u[..., odd] = pairs.real, pairs.imag
            if c["norm"]:
                dg += (u * z).sum((0, 1))
                u = u * gain
                u = (u - z * ((u * z).sum(2, keepdim=True) / d)) / root
            dx[rows] = u
        out[x] = y
        if grads is not None:
            out["d" + x] = dx
            if c["norm"]:
                out["dg" + x] = dg
    return out


def _exact_read(c, s):
    """A sequence at a time."""
    k, v = (torch.empty(s["k_out"].shape, dtype=torch.float64, device=DEV) for _ in range(2))
    row = 0
    for i, (n, total) in enumerate(zip(*_lengths(c))):
        first = (total - n) // PAGE
        pages = s["table"][i, first:-(-total // PAGE)].long()
        a = total - n - first * PAGE
        for codes, scale, out, by_token in ((s["k"], s["ks"], k, True), (s["v"], s["vs"], v, False)):
            x = codes.view(torch.uint8)[pages].view(F8).to(torch.float64) * scale[pages].to(torch.float64)[:, :, None, None]
            x = x.permute(0, 2, 1, 3) if by_token else x.permute(0, 3, 1, 2)
            out[row:row + n] = x.reshape(-1, c["hkv"], c["d"])[a:a + n]
        row += n
    return {"k": k, "v": v}


def _exact_shared(c, s):
    """Head by head, a sequence at a time over all of its tokens."""
    f64, hkv, d, g = torch.float64, c["hkv"], c["d"], c["hq"] // c["hkv"]
    members, prefix, n, tails = _groups(c)
    lens = (np.repeat(prefix, members) + tails).tolist()
    if sum(lens) * c["hq"] * d > 3e11:
        return None
    o, lse = torch.zeros(s["q"].shape, dtype=f64, device=DEV), torch.zeros(c["hq"], s["q"].shape[0], dtype=f64, device=DEV)
    row = 0
    for i, (r, total) in enumerate(zip(n, lens)):
        pages = s["table"][i, :-(-total // PAGE)].long()
        hidden = torch.arange(total, device=DEV) > torch.arange(total - r, total, device=DEV)[:, None]
        for h in range(hkv):
            k = (s["k"][:, h].view(torch.uint8)[pages].view(F8).to(f64) * s["ks"][pages, h].to(f64)[:, None, None]).reshape(-1, d)[:total]
            v = (s["v"][:, h].view(torch.uint8)[pages].view(F8).to(f64) * s["vs"][pages, h].to(f64)[:, None, None]).transpose(1, 2).reshape(-1, d)[:total]
            q = s["q"][row:row + r, h * g:(h + 1) * g].to(f64).transpose(0, 1)
            x = ((q.reshape(g * r, d) @ k.t().contiguous()) / math.sqrt(d)).view(g, r, total).masked_fill_(hidden, -math.inf)
            whole = torch.logsumexp(x, 2)
            o[row:row + r, h * g:(h + 1) * g] = ((x - whole[:, :, None]).exp_().view(g * r, total) @ v).view(g, r, d).transpose(0, 1)
            lse[h * g:(h + 1) * g, row:row + r] = whole
        row += r
    return {"o": o, "lse": lse}
