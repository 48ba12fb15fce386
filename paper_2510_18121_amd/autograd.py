"""torch.autograd wrapper over the C-ABI calls, for training code that wants an attention-server step as one
differentiable op (the paper's runtime calls a fused variable-length attention kernel per server step, Section 4.1;
this is the same call shape: packed Q, K, V in, packed O out, gradients through backward()).

Plumbing only: forward() calls ca_forward, backward() calls ca_backward; nothing is computed here.  The op saves
Q, K, V, O and the per-row log-sum-exp and recomputes P in backward (Section 2.1)."""
from __future__ import annotations

import numpy as np
import torch

from . import binding as B
from .rotary import GAP


class _CoreAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, server):
        b = server.plan.batch
        o = torch.empty_like(q)
        lse = torch.empty((b.n_q_heads, b.total_q), dtype=torch.float32, device=q.device)
        # partial results of the forward have memory of the call's own: forwards of one server may overlap in time (other
        # streams, or another call's backward, which uses the server's workspace)
        B.ca_forward(server.plan, q, k, v, o, lse, B._scratch(server.fwd_ws_bytes, 0, q.device))
        ctx.save_for_backward(q, k, v, o, lse)
        ctx.server = server
        return o

    @staticmethod
    def backward(ctx, d_o):
        q, k, v, o, lse = ctx.saved_tensors
        s = ctx.server
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        d_o = d_o.contiguous()
        if d_o.data_ptr() % 16 != 0:  # (where autograd's tensors lie is not the caller's choice)
            d_o = d_o.clone()
        B.ca_backward(s.plan, q, k, v, o, d_o, lse, dq, dk, dv, s.ws)
        return dq, dk, dv, None


def row_positions(batch):
    """Document position of every row of the packed Q, and of the packed K (int32; 0 for rows of no task, keys of no document)."""
    q, kv = np.zeros(batch.total_q, np.int32), np.zeros(batch.total_kv, np.int32)
    for rows, starts, lens, first in ((q, batch.task_q_start, batch.task_q_len, batch.task_q_pos),
                                      (kv, batch.doc_kv_start, batch.doc_kv_len, np.zeros(len(batch.doc_kv_len), np.int64))):
        for a, n, p in zip(*(np.asarray(x).tolist() for x in (starts, lens, first))):
            rows[a:a + n] = np.arange(p, p + n)
    return q, kv


def rows_in_use(batch, window=None, sinks=0):
    """Which rows of the packed Q belong to a task, and which of the packed K some row of a task sees."""
    q, kv = np.zeros(batch.total_q, bool), np.zeros(batch.total_kv, bool)
    for doc, a, n, p, length in zip(*(np.asarray(x).tolist() for x in (batch.task_doc, batch.task_q_start, batch.task_q_len, batch.task_q_pos, batch.task_kv_len))):
        if n > 0:
            q[a:a + n] = True
            first, end = int(batch.doc_kv_start[doc]), min(p + n, length)  # (the last row sees end tokens, the first row's window begins furthest back)
            begin = 0 if window is None else min(max(0, p - window + 1), end)
            kv[first + begin:first + end] = kv[first:first + min(sinks, end)] = True
    return q, kv


class AttentionServer:
    """One fused batch of CA-tasks planned once and run as a differentiable op:

        server = AttentionServer(batch)          # plans, uploads, allocates the workspace
        o = server(q, k, v)                      # bf16 [total_q, Hq, D]; q, k, v may require grad
        o.backward(d_o)                          # q.grad, k.grad, v.grad

    `batch` is any object with the descriptor's fields (e.g. workloads.Batch).  Rows of q that belong to no task
    have undefined output and zero gradient.  one_pass: see binding.alloc_workspace.  window, sinks: every row attends the last
    `window` keys of its context, itself among them, and the context's first `sinks` (None: all of it); see binding.ca_plan.
    rotation (rotary.Rotation): q and k are turned by the positions of their rows in their documents first, and, with gains, each head of
    them is normed before: o = server(q, k, v, q_gain, k_gain).  Rows that no task has, and keys that none sees, add nothing to the gradients
    of the gains, whatever they hold."""

    def __init__(self, batch, device="cuda", one_pass=None, window=None, sinks=0, rotation=None, eps=1e-6):
        if rotation is not None and rotation.head_dim != batch.head_dim:
            raise ValueError(f"the rotation's head_dim is {rotation.head_dim}, the batch's {batch.head_dim}")
        self.plan = B.ca_plan(batch, window, sinks)
        self.ws = B.alloc_workspace(self.plan, device, one_pass)
        self.fwd_ws_bytes = self.plan.workspace_bytes_split()[0]
        self.rotation, self.eps = rotation, eps
        if rotation is not None:
            positions = row_positions(batch)
            self.q_pos, self.kv_pos = (torch.from_numpy(x).to(device) for x in positions)
            self.grad_pos = [None if used.all() else torch.from_numpy(np.where(used, x, GAP).astype(np.int32)).to(device)
                             for x, used in zip(positions, rows_in_use(batch, window, sinks))]

    def __call__(self, q, k, v, q_gain=None, k_gain=None):
        if self.rotation is not None:
            q, k = self.rotation(q, k, self.q_pos, self.kv_pos, q_gain=q_gain, k_gain=k_gain, eps=self.eps, grad_pos=self.grad_pos)
        elif q_gain is not None or k_gain is not None:
            raise ValueError("gains without a rotation (one of no frequencies turns nothing)")
        return _CoreAttention.apply(q, k, v, self)
