"""Queries and keys on their way to attention: turned by their positions, each head normed before (or not), and their gradients.

    rotation = Rotation(head_dim, base=500000.0)                         # half layout, the whole head
    q, k = rotation(q, k, q_pos)                                         # bf16 [rows, heads, head_dim], int32 [rows]; differentiable
    q, k = rotation(q, k, q_pos, k_pos, q_gain=gq, k_gain=gk, eps=1e-6)  # the norm of each head first, with learnt gains [head_dim]
    server = AttentionServer(batch, rotation=rotation)                   # ... as a part of the attention of a batch of CA-tasks

For new tokens of cached sequences binding.ca_rotate takes the positions from the arrays of cache.Sequences.  Frequencies for contexts
longer than those that a model was trained on: `interpolated`, `by_parts`, or any array of radians per position.

Plumbing only: what is computed runs in the library's kernels (include/ca_attention.h)."""
from __future__ import annotations

import ctypes
import math
import operator
from fractions import Fraction

import numpy as np
import torch

GAP = -2 ** 31  # the position of a row that takes no part in a gradient (see Rotation.__call__)
TWO_PI = 2 * Fraction(314159265358979323846264338327950288419716939937510, 10 ** 50)


class RotationDesc(ctypes.Structure):
    """ca_rotation of include/ca_attention.h."""

    _fields_ = [("head_dim", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("factor", ctypes.c_float),
                ("turns", ctypes.c_void_p)]


def frequencies(rot_dim, base=10000.0):
    """Radians per position of the rot_dim / 2 pairs: base^(-2 i / rot_dim)."""
    rot_dim = operator.index(rot_dim)
    if rot_dim < 0 or rot_dim % 2 or not base > 0:
        raise ValueError(f"rot_dim {rot_dim}, base {base}: an even number, and positive")
    return float(base) ** (-2 * np.arange(rot_dim // 2) / max(rot_dim, 1))


def interpolated(freq, factor):
    """Frequencies for contexts `factor` times as long: all of them slowed down."""
    if not factor > 0:
        raise ValueError(f"factor {factor}: positive")
    return np.asarray(freq, np.float64) / factor


def by_parts(freq, factor, trained_length, slow=1.0, fast=32.0):
    """Frequencies for contexts `factor` times as long as trained_length: pairs that turn at most `slow` times in that length are slowed down, those that
    turn at least `fast` times are kept, and the ones between are mixed in proportion to their turns."""
    freq = np.asarray(freq, np.float64)
    if not (factor > 0 and trained_length > 0 and 0 <= slow < fast):
        raise ValueError(f"factor {factor}, trained_length {trained_length}, slow {slow}, fast {fast}: positive, and slow below fast")
    kept = np.clip((trained_length * np.abs(freq) / (2 * math.pi) - slow) / (fast - slow), 0, 1)
    return freq * (kept + (1 - kept) / factor)


class Rotation:
    """How heads are turned: rot_dim (the first columns of a head, all of them by default) and base, or `frequencies` (radians per position
    of each pair, in which case rot_dim is twice their number; none: nothing is turned); interleaved: pairs (2 i, 2 i + 1), otherwise
    (i, i + rot_dim / 2); factor: of the turned columns."""

    def __init__(self, head_dim, rot_dim=None, base=10000.0, frequencies=None, interleaved=False, factor=1.0, device="cuda"):
        head_dim = operator.index(head_dim)
        if head_dim not in (64, 128):
            raise ValueError(f"head_dim {head_dim}: 64 or 128")
        if frequencies is None:
            frequencies = globals()["frequencies"](head_dim if rot_dim is None else rot_dim, base)
        freq = np.asarray(frequencies, np.float64)
        if freq.ndim != 1 or 2 * freq.size > head_dim or (rot_dim is not None and 2 * freq.size != operator.index(rot_dim)):
            raise ValueError(f"frequencies: {freq.shape}, expected [rot_dim / 2], at most [{head_dim // 2}]")
        if not np.isfinite(freq).all() or not math.isfinite(factor):
            raise ValueError("frequencies and factor: finite numbers")
        turns = np.array([round(Fraction(f) / TWO_PI * 2 ** 64) % 2 ** 64 for f in freq.tolist()], np.uint64)
        self.head_dim, self.rot_dim, self.interleaved, self.factor = head_dim, 2 * freq.size, bool(interleaved), float(factor)
        self.frequencies = freq
        self.turns = torch.from_numpy(turns.view(np.int64)).to(device)
        self._describe()

    def _describe(self):
        """What belongs to this process and to where `turns` lies."""
        self.device = self.turns.device
        self.desc = RotationDesc(self.head_dim, self.rot_dim, self.interleaved, self.factor, self.turns.data_ptr() if self.rot_dim else None)
        self.desc_ref = ctypes.byref(self.desc)
        # what the calls look up every time
        self.index = self.turns.get_device() if self.turns.is_cuda else None  # (None: no tensor is there)
        self.i32, self.f32, self.bf16 = torch.int32, torch.float32, torch.bfloat16
        # (where there is a tensor on a device it is initialised, which is what torch.cuda.current_device looks at first)
        self.current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        self.raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)

    def __getstate__(self):  # (copied and saved with the module that holds it)
        return {x: getattr(self, x) for x in ("head_dim", "rot_dim", "interleaved", "factor", "frequencies", "turns")}

    def __setstate__(self, state):
        self.__dict__.update(state)
        self._describe()

    def __call__(self, q, k=None, q_pos=None, k_pos=None, where=None, q_gain=None, k_gain=None, eps=1e-6, grad_pos=(None, None)):
        """q and k [rows, heads, head_dim] (bf16; k may be None), turned, as contiguous tensors; differentiable in q, k and the gains (fp32
        or bf16 [head_dim]).  Positions: q_pos and k_pos (int32 [rows]; k_pos None: those of q), or where = (q_start, kv_len, ..) of sequences
        (see binding.ca_rotate).  Rows of no sequence are undefined, and their gradients zero.  grad_pos: of q and of k, None or the same positions (int32
        [rows]) but GAP at rows that have no gradient, whatever they hold: theirs are zero, and they add nothing to the gains'.  A training pass is captured into a graph with
        torch.autograd.grad, while no eager graph of the same leaves lives."""
        gains = [None if g is None else g.float().contiguous() for g in (q_gain, k_gain)]
        q_start, kv_len = (None, None) if where is None else where[:2]
        out = _Rotate.apply(q, k, *gains, self, q_pos, k_pos, q_start, kv_len, float(eps), *grad_pos)
        return out if k is not None else out[0]


class _Rotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_gain, k_gain, rotation, q_pos, k_pos, q_start, kv_len, eps, q_grad_pos, k_grad_pos):
        from . import binding as B
        yq, yk = (None if x is None else torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k))
        B.ca_rotate(rotation, q, k, yq, yk, q_pos, k_pos, None if q_start is None else (q_start, kv_len), q_gain, k_gain, eps)
        ctx.gaps = q_grad_pos is not None, k_grad_pos is not None
        k_pos = k_grad_pos if k_grad_pos is not None else q_pos if k_pos is None else k_pos
        q_pos = q_pos if q_grad_pos is None else q_grad_pos
        # (without a gain the gradient needs no input)
        ctx.save_for_backward(*(x if g is not None else None for x, g in ((q, q_gain), (k, k_gain))), q_gain, k_gain, q_pos, k_pos, q_start, kv_len)
        ctx.rotation, ctx.eps = rotation, eps
        return yq, yk

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dyq, dyk):
        from . import binding as B
        q, k, q_gain, k_gain, q_pos, k_pos, q_start, kv_len = ctx.saved_tensors
        where = None if q_start is None else (q_start, kv_len)
        dys = [None if d is None else B.rows_in_line(d) for d in (dyq, dyk)]
        # (zeros: rows of no sequence, and gaps)
        dx = [None if d is None else (torch.empty if where is None and not gaps else torch.zeros)(d.shape, dtype=d.dtype, device=d.device)
              for d, gaps in zip(dys, ctx.gaps)]
        dg = [None if g is None else torch.empty_like(g) for g in (q_gain, k_gain)]
        ws = B.alloc_rotate_workspace(dys[0].device) if q_gain is not None or k_gain is not None else None
        B.ca_rotate_backward(ctx.rotation, q, k, *dys, *dx, q_pos, k_pos, where, q_gain, k_gain, *dg, ctx.eps, ws, None, *ctx.gaps)
        return *dx, *dg, *[None] * 8
