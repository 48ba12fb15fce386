"""A paged cache of keys and values in 8 bits, and the host's book-keeping of its pages.

`KVCache` is the device memory of one layer's cache (see include/ca_attention.h for the layout); binding.ca_cache_append,
ca_cache_attend and ca_cache_copy_pages work on it.  `Sequences` says which pages belong to which sequence: it hands pages out, shares
them between forks, copies a shared page before it is written, frees the pages that a window has left behind, and compacts the pool.
One `Sequences` serves the caches of all layers, which then hold a token in the same page.

    cache = KVCache.empty(n_pages, n_kv_heads, head_dim)
    seqs = Sequences([cache])
    ws = binding.alloc_cache_workspace(cache, n_q_heads)
    a = seqs.add()
    q_start, kv_len, table = seqs.extend([a], [len(prompt)])           # room for the rows, and where they are
    binding.ca_cache_append(cache, k, v, q_start, kv_len, table)       # bf16 [rows, n_kv_heads, head_dim]
    binding.ca_cache_attend(cache, q, o, lse, q_start, kv_len, table, ws)
"""
from __future__ import annotations

import ctypes
import operator

import numpy as np

PAGE_TOKENS = 64


class CacheDesc(ctypes.Structure):
    """ca_cache of include/ca_attention.h."""

    _fields_ = [("n_pages", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class KVCache:
    """k: e4m3 [n_pages, n_kv_heads, 64, head_dim], v: e4m3 [n_pages, n_kv_heads, head_dim, 64], k_scale and v_scale: fp32
    [n_pages, n_kv_heads], contiguous tensors of one device."""

    def __init__(self, k, v, k_scale, v_scale):
        import torch
        pages, heads, tokens, dim = k.shape
        for t, shape, dtype, name in ((k, (pages, heads, PAGE_TOKENS, dim), torch.float8_e4m3fn, "k"),
                                      (v, (pages, heads, dim, PAGE_TOKENS), torch.float8_e4m3fn, "v"),
                                      (k_scale, (pages, heads), torch.float32, "k_scale"), (v_scale, (pages, heads), torch.float32, "v_scale")):
            if t.shape != shape or t.dtype != dtype or not t.is_contiguous() or t.device != k.device:
                raise ValueError(f"{name}: expected contiguous tensor {shape} {dtype} on {k.device}, got {tuple(t.shape)} {t.dtype} on {t.device}")
        if dim not in (64, 128):
            raise ValueError(f"head_dim {dim}: 64 or 128")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.n_kv_heads, self.head_dim, self.device = pages, heads, dim, k.device
        self.desc = CacheDesc(pages, heads, dim, *(t.data_ptr() if pages else None for t in (k, v, k_scale, v_scale)))
        self.desc_ref = ctypes.byref(self.desc)
        # what the calls look up every time
        self.index = k.get_device() if k.is_cuda else None  # (None: no tensor is there)
        self.i32, self.f32, self.bf16 = torch.int32, torch.float32, torch.bfloat16
        self.current_device, self.raw_stream = torch.cuda.current_device, getattr(torch._C, "_cuda_getCurrentRawStream", None)

    @classmethod
    def empty(cls, n_pages, n_kv_heads, head_dim, device="cuda"):
        """A cache of pages that hold nothing yet."""
        import torch
        f8, f32 = torch.float8_e4m3fn, torch.float32
        return cls(torch.empty(n_pages, n_kv_heads, PAGE_TOKENS, head_dim, dtype=f8, device=device),
                   torch.empty(n_pages, n_kv_heads, head_dim, PAGE_TOKENS, dtype=f8, device=device),
                   *(torch.empty(n_pages, n_kv_heads, dtype=f32, device=device) for _ in range(2)))


class OutOfPages(RuntimeError):
    """The pool has fewer free pages than a call needs."""


class Sequences:
    """The pages of sequences in a pool of n_pages (the fewest that one of `caches` has, unless fewer are given; without caches nothing is
    copied on a device)."""

    def __init__(self, caches=(), n_pages=None):
        self.caches = list(caches)
        if n_pages is None:
            n_pages = min(c.n_pages for c in self.caches)
        if operator.index(n_pages) < 0 or any(c.n_pages < n_pages for c in self.caches):
            raise ValueError(f"n_pages {n_pages}: not negative, and no more than each of the caches has")
        self.free_pages = list(range(n_pages - 1, -1, -1))  # the lowest is handed out first
        self.uses = [0] * n_pages                           # sequences that hold the page
        self.pages, self.lengths = {}, {}                   # of each sequence; a page that was let go is -1
        self._next = 0

    def add(self):
        """A new sequence without tokens."""
        self._next += 1
        self.pages[self._next], self.lengths[self._next] = [], 0
        return self._next

    def fork(self, seq):
        """A new sequence with the tokens of `seq`, on the same pages."""
        new = self.add()
        self.pages[new], self.lengths[new] = list(self.pages[seq]), self.lengths[seq]
        for p in self.pages[new]:
            if p >= 0:
                self.uses[p] += 1
        return new

    def free(self, seq):
        """Gives a sequence's pages back."""
        for p in self.pages.pop(seq):
            self._let_go(p)
        del self.lengths[seq]

    def leave_window(self, seq, window, sinks=0):
        """Gives back the pages that no later row of `seq` sees with that window and those sinks."""
        if operator.index(window) < 1 or operator.index(sinks) < 0:
            raise ValueError(f"window {window}, sinks {sinks}: at least 1, and not negative")
        pages = self.pages[seq]
        for i in range(-(-sinks // PAGE_TOKENS), min(max(0, self.lengths[seq] - window + 1) // PAGE_TOKENS, len(pages))):
            self._let_go(pages[i])
            pages[i] = -1

    def extend(self, seqs, rows, device=None):
        """Room for rows[i] more tokens of seqs[i], and the call's arrays: q_start, kv_len and page_table on the device.  A last page that
        other sequences hold too is copied for each of them first.  On the current stream.  Where it raises, nothing has changed."""
        seqs, rows = list(seqs), [operator.index(n) for n in rows]
        if len(seqs) != len(rows) or len(set(seqs)) != len(seqs) or any(n < 0 for n in rows):
            raise ValueError("extend: one count of rows, not negative, for each of the sequences, and each of them once")
        need, copies, taken = 0, [], {}
        for s, n in zip(seqs, rows):
            held = self.lengths[s]
            need += -(-(held + n) // PAGE_TOKENS) - len(self.pages[s])
            if n and held % PAGE_TOKENS:
                p = self.pages[s][-1]
                if p < 0:
                    raise ValueError("extend: the last page has been let go")
                if self.uses[p] - taken.get(p, 0) > 1:
                    taken[p] = taken.get(p, 0) + 1
                    copies.append(s)
        if need + len(copies) > len(self.free_pages):
            raise OutOfPages(f"{need + len(copies)} pages needed, {len(self.free_pages)} free")
        # what may fail comes before what changes
        free = iter(self.free_pages[::-1])
        pages = {s: list(self.pages[s]) for s in seqs}
        src = [pages[s][-1] for s in copies]
        for s in copies:
            pages[s][-1] = next(free)
        dst = [pages[s][-1] for s in copies]
        for s, n in zip(seqs, rows):
            pages[s] += [next(free) for _ in range(-(-(self.lengths[s] + n) // PAGE_TOKENS) - len(pages[s]))]
        self._copy(src, dst)
        out = self._arrays([pages[s] for s in seqs], [self.lengths[s] + n for s, n in zip(seqs, rows)], rows, device)
        for _ in range(need + len(copies)):
            self.uses[self.free_pages.pop()] = 1
        for p in src:
            self._let_go(p)
        for s, n in zip(seqs, rows):
            self.pages[s] = pages[s]
            self.lengths[s] += n
        return out

    def arrays(self, seqs, rows, device=None):
        """q_start, kv_len and page_table (int32) of a call with the last rows[i] tokens of seqs[i]."""
        return self._arrays([self.pages[s] for s in seqs], [self.lengths[s] for s in seqs], rows, device)

    def _arrays(self, pages, lengths, rows, device):
        import torch
        table = np.full((len(pages), max([len(x) for x in pages], default=0)), -1, np.int32)
        for i, x in enumerate(pages):
            table[i, :len(x)] = x
        start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        if device is None:
            device = self.caches[0].device if self.caches else "cpu"
        return tuple(torch.from_numpy(x).to(device) for x in (start, np.array(lengths, np.int32), table))

    def compact(self):
        """Moves the pages in use to the front of the pool, on the current stream; returns how many are in use.  Page tables made before are
        out of date."""
        n = sum(u > 0 for u in self.uses)
        holes = [p for p in range(n) if self.uses[p] == 0]
        moved = dict(zip([p for p in range(n, len(self.uses)) if self.uses[p]], holes))
        self._copy(list(moved), list(moved.values()))
        for pages in self.pages.values():
            pages[:] = [moved.get(p, p) for p in pages]
        for p, to in moved.items():
            self.uses[to], self.uses[p] = self.uses[p], 0
        self.free_pages = list(range(len(self.uses) - 1, n - 1, -1))
        return n

    def _let_go(self, p):
        if p >= 0:
            self.uses[p] -= 1
            if self.uses[p] == 0:
                self.free_pages.append(p)

    def _copy(self, src, dst):
        if not src:
            return
        import torch

        from . import binding as B
        for c in self.caches:
            B.ca_cache_copy_pages(c, *(torch.tensor(x, dtype=torch.int32, device=c.device) for x in (src, dst)))
