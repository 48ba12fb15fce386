"""Thin Python binding over the C ABI of libca_attention.so (include/ca_attention.h).

Argument marshalling only: every step of the path runs inside the library's HIP kernels.  PyTorch
tensors are used as device memory and streams and nothing else.  There is no fallback: if the
library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import operator
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libca_attention.so")
_lib = None

CA_OK = 0
CA_ERR_INVALID_ARG, CA_ERR_UNSUPPORTED, CA_ERR_WORKSPACE, CA_ERR_HIP, CA_ERR_STATE = -1, -2, -3, -4, -5


class CaError(RuntimeError):
    """A negative ca_status from the library, with its code and the library's detail string."""

    def __init__(self, code: int, detail: str):
        super().__init__(f"ca_attention error {code}: {detail}")
        self.code = code
        self.detail = detail


class BatchDesc(ctypes.Structure):
    """ca_batch_desc of include/ca_attention.h."""

    _fields_ = [
        ("n_docs", ctypes.c_int32), ("n_tasks", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("total_q", ctypes.c_int64), ("total_kv", ctypes.c_int64), ("softmax_scale", ctypes.c_float),
        ("doc_kv_start", ctypes.c_void_p), ("doc_kv_len", ctypes.c_void_p), ("task_doc", ctypes.c_void_p),
        ("task_q_start", ctypes.c_void_p), ("task_q_len", ctypes.c_void_p), ("task_q_pos", ctypes.c_void_p),
        ("task_kv_len", ctypes.c_void_p),
    ]


class CacheBatch(ctypes.Structure):
    """ca_cache_batch of include/ca_attention.h."""

    _fields_ = [("n_seqs", ctypes.c_int32), ("table_width", ctypes.c_int32), ("total_rows", ctypes.c_int64),
                ("q_start", ctypes.c_void_p), ("kv_len", ctypes.c_void_p), ("page_table", ctypes.c_void_p)]


class CacheGroups(ctypes.Structure):
    """ca_cache_groups of include/ca_attention.h."""

    _fields_ = [("n_groups", ctypes.c_int32), ("group_start", ctypes.c_void_p), ("prefix_pages", ctypes.c_void_p)]


class RotateTensor(ctypes.Structure):
    """ca_rotate_tensor of include/ca_attention.h."""

    _fields_ = [("x", ctypes.c_void_p), ("dy", ctypes.c_void_p), ("y", ctypes.c_void_p), ("gain", ctypes.c_void_p), ("dgain", ctypes.c_void_p),
                ("pos", ctypes.c_void_p), ("rows", ctypes.c_int64), ("x_stride", ctypes.c_int64), ("dy_stride", ctypes.c_int64),
                ("y_stride", ctypes.c_int64), ("heads", ctypes.c_int32), ("gaps", ctypes.c_int32)]


def lib() -> ctypes.CDLL:
    """The loaded C-ABI library; raises if it has not been built (python -m paper_2510_18121_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                                    "or python paper_2510_18121_amd/build.py")
        L = ctypes.CDLL(LIB_PATH)
        vp, sz = ctypes.c_void_p, ctypes.c_size_t
        L.ca_plan_host.argtypes = [ctypes.POINTER(BatchDesc), ctypes.POINTER(vp)]
        L.ca_plan.argtypes = [ctypes.POINTER(BatchDesc), ctypes.POINTER(vp)]
        for f in (L.ca_plan_window, L.ca_plan_window_host):
            f.argtypes = [ctypes.POINTER(BatchDesc), ctypes.c_int64, ctypes.c_int64, ctypes.POINTER(vp)]
        L.ca_plan_window_units.argtypes = [vp, ctypes.c_int32, vp]
        L.ca_plan_upload.argtypes = [vp, vp]
        L.ca_plan_workspace_bytes.argtypes = [vp, ctypes.POINTER(sz), ctypes.POINTER(sz)]
        L.ca_plan_workspace_bytes_split.argtypes = [vp, ctypes.POINTER(sz), ctypes.POINTER(sz)]
        L.ca_forward.argtypes = [vp] * 6 + [vp, sz, vp]
        L.ca_backward.argtypes = [vp] * 10 + [vp, sz, vp]
        L.ca_backward_static_ws.argtypes = [vp] * 10 + [vp]
        L.ca_static_workspace_bytes.restype = sz
        L.ca_plan_destroy.argtypes = [vp]
        L.ca_plan_destroy.restype = None
        L.ca_error_string.argtypes = [ctypes.c_int]
        L.ca_error_string.restype = ctypes.c_char_p
        L.ca_last_error.restype = ctypes.c_char_p
        L.ca_profile_enable.argtypes = [vp, ctypes.c_int]
        L.ca_profile_read.argtypes = [vp, vp]
        L.ca_plan_info.argtypes = [vp, vp, ctypes.c_int]
        for f in (L.ca_plan_rows, L.ca_plan_fwd_units, L.ca_plan_bwd_units, L.ca_plan_fwd_pieces, L.ca_plan_bwd_pieces,
                  L.ca_plan_combine_units, L.ca_plan_one_pass_units, L.ca_plan_window_units):
            f.restype = ctypes.c_int64
        L.ca_plan_fwd_pieces.argtypes = [vp, vp]
        L.ca_plan_bwd_pieces.argtypes = [vp, vp, vp]
        L.ca_plan_workspace_bytes_one_pass.argtypes = [vp, vp]
        L.ca_plan_one_pass_units.argtypes = [vp, vp, vp]
        L.ca_plan_combine_units.argtypes = [vp, ctypes.c_int32, vp]
        L.ca_plan_rows.argtypes = [vp, vp, vp]
        L.ca_plan_fwd_units.argtypes = [vp, vp]
        L.ca_plan_bwd_units.argtypes = [vp, vp]
        i32, i64 = ctypes.c_int32, ctypes.c_int64
        L.ca_merge_partials.argtypes = [vp, i64, i32, vp, vp, i64, vp, vp, vp, vp, i32, i32, vp]
        L.ca_sum_partial_dq.argtypes = [vp, i64, i32, vp, i64, vp, i32, i32, vp]
        L.ca_cache_append.argtypes = [vp] * 5
        L.ca_cache_read.argtypes = [vp] * 5
        L.ca_cache_attend_shared.argtypes = [vp, vp, vp, i32, ctypes.c_float, vp, vp, vp, vp, sz, vp]
        L.ca_cache_attend_shared_workspace_bytes.argtypes = [vp, i32, i64, ctypes.POINTER(sz)]
        L.ca_cache_attend.argtypes = [vp, vp, i32, ctypes.c_float, i64, i64, vp, vp, vp, vp, sz, vp]
        L.ca_cache_attend_workspace_bytes.argtypes = [vp, i32, ctypes.POINTER(sz)]
        L.ca_cache_copy_pages.argtypes = [vp, vp, vp, i64, vp]
        L.ca_rotate.argtypes = [vp, vp, i32, vp, ctypes.c_float, vp]
        L.ca_rotate_backward.argtypes = [vp, vp, i32, vp, ctypes.c_float, vp, sz, vp]
        L.ca_rotate_backward_workspace_bytes.restype = sz
        L.ca_mfma_stream.argtypes = L.ca_mfma_stream16.argtypes = [vp, i64, i32, i32, vp, vp]
        L.ca_xcd_map.argtypes = [i32, i32, vp, vp]
        L.ca_atomic_stream.argtypes = [vp, vp, i32, i32, i32, i32, i32, vp, vp]
        _lib = L
    return _lib


def _check(rc: int):
    if rc != CA_OK:
        raise CaError(rc, (lib().ca_last_error() or b"").decode())


def make_desc(batch, keep: list) -> BatchDesc:
    """ca_batch_desc from any object with the descriptor's field names (e.g. workloads.Batch)."""
    def arr(x, dt):
        a = np.ascontiguousarray(np.asarray(x), dtype=dt)
        keep.append(a)
        return a.ctypes.data if a.size else None

    d = BatchDesc()
    d.n_docs, d.n_tasks = len(batch.doc_kv_len), len(batch.task_q_len)
    d.n_q_heads, d.n_kv_heads, d.head_dim = batch.n_q_heads, batch.n_kv_heads, batch.head_dim
    d.total_q, d.total_kv, d.softmax_scale = batch.total_q, batch.total_kv, float(batch.softmax_scale)
    d.doc_kv_start = arr(batch.doc_kv_start, np.int64)
    d.doc_kv_len = arr(batch.doc_kv_len, np.int64)
    d.task_doc = arr(batch.task_doc, np.int32)
    d.task_q_start = arr(batch.task_q_start, np.int64)
    d.task_q_len = arr(batch.task_q_len, np.int64)
    d.task_q_pos = arr(batch.task_q_pos, np.int64)
    d.task_kv_len = arr(batch.task_kv_len, np.int64)
    return d


class Plan:
    """Owner of a ca_plan_t*."""

    INFO_KEYS = ("q_tile_rows", "n_q_tiles", "n_fwd_units", "kv_tile_rows", "n_bwd_units", "fwd_kv_step",
                 "padded_rows", "fwd_steps", "bwd_steps", "bwd_q_block_rows", "slot_align", "heads_packed",
                 "n_bwd_workgroups", "joint_backward", "forward_halves", "forward_piece_halves",
                 "forward_turns", "forward_piece_turns", "one_pass_backward")

    def __init__(self, handle, batch):
        self.handle = ctypes.c_void_p(handle)
        self.batch = batch

    def upload(self, stream=None):
        _check(lib().ca_plan_upload(self.handle, _stream_ptr(stream)))
        return self

    def workspace_bytes(self):
        f, b = ctypes.c_size_t(), ctypes.c_size_t()
        _check(lib().ca_plan_workspace_bytes(self.handle, ctypes.byref(f), ctypes.byref(b)))
        return int(f.value), int(b.value)

    def workspace_bytes_split(self):
        """Workspace (forward, backward) with which the calls also cut long units into pieces."""
        f, b = ctypes.c_size_t(), ctypes.c_size_t()
        _check(lib().ca_plan_workspace_bytes_split(self.handle, ctypes.byref(f), ctypes.byref(b)))
        return int(f.value), int(b.value)

    def workspace_bytes_one_pass(self):
        """Workspace with which the backward runs in one pass; 0 where that would not be faster."""
        b = ctypes.c_size_t()
        _check(lib().ca_plan_workspace_bytes_one_pass(self.handle, ctypes.byref(b)))
        return int(b.value)

    def info(self) -> dict:
        out = np.zeros(len(self.INFO_KEYS), np.int64)
        lib().ca_plan_info(self.handle, out.ctypes.data, len(out))
        return dict(zip(self.INFO_KEYS, out.tolist()))

    def rows(self):
        n = lib().ca_plan_rows(self.handle, None, None)
        r, p = np.zeros(n, np.int32), np.zeros(n, np.int32)
        lib().ca_plan_rows(self.handle, r.ctypes.data, p.ctypes.data)
        return r, p

    def fwd_units(self):
        n = lib().ca_plan_fwd_units(self.handle, None)
        u = np.zeros((n, 5), np.int32)
        lib().ca_plan_fwd_units(self.handle, u.ctypes.data)
        return u

    def bwd_units(self):
        n = lib().ca_plan_bwd_units(self.handle, None)
        u = np.zeros((n, 10), np.int32)
        lib().ca_plan_bwd_units(self.handle, u.ctypes.data)
        return u

    def window_units(self):
        """Forward units, dK/dV units and the slots' windows of a windowed plan (arrays as in the header; empty for any other)."""
        out = []
        for kind, fields in ((0, 8), (1, 12), (2, 1)):
            out.append(np.zeros((lib().ca_plan_window_units(self.handle, kind, None), fields), np.int32))
            lib().ca_plan_window_units(self.handle, kind, out[-1].ctypes.data)
        return out[0], out[1], out[2][:, 0]

    def one_pass_units(self):
        """Units of the backward in one pass (fields as in bwd_units), and where each XCD's queue of them begins."""
        n = lib().ca_plan_one_pass_units(self.handle, None, None)
        u, q = np.zeros((n, 10), np.int32), np.zeros(9, np.int32)
        lib().ca_plan_one_pass_units(self.handle, u.ctypes.data, q.ctypes.data)
        return u, q

    def pieces(self) -> dict:
        """The lists of units cut into pieces (arrays as in the header; empty where nothing is cut)."""
        L, n_wg = lib(), ctypes.c_int32()
        fwd = np.zeros((L.ca_plan_fwd_pieces(self.handle, None), 8), np.int32)
        L.ca_plan_fwd_pieces(self.handle, fwd.ctypes.data)
        bwd = np.zeros((L.ca_plan_bwd_pieces(self.handle, None, None), 10), np.int32)
        L.ca_plan_bwd_pieces(self.handle, bwd.ctypes.data, ctypes.byref(n_wg))
        out = {"fwd": fwd, "bwd": bwd, "bwd_workgroups": n_wg.value}
        for key, backward in (("fwd_combine", 0), ("bwd_combine", 1)):
            out[key] = np.zeros((L.ca_plan_combine_units(self.handle, backward, None), 6), np.int32)
            L.ca_plan_combine_units(self.handle, backward, out[key].ctypes.data)
        return out

    def profile_enable(self, on=True):
        _check(lib().ca_profile_enable(self.handle, 1 if on else 0))

    def profile_read(self) -> dict:
        out = np.zeros(4, np.float32)
        _check(lib().ca_profile_read(self.handle, out.ctypes.data))
        return dict(zip(("fwd_kernel_ms", "bwd_prep_ms", "bwd_dkv_ms", "bwd_dq_ms"), out.tolist()))

    def destroy(self):
        if self.handle:
            lib().ca_plan_destroy(self.handle)
            self.handle = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def _count(x) -> int:
    """An integer for an int64 argument, where ctypes would take it modulo 2^64; beyond 2^63 - 1 one is as good as another."""
    return max(-1, min(operator.index(x), (1 << 63) - 1))


def _planned(batch, window, sinks, plain, windowed) -> Plan:
    keep = []
    d = make_desc(batch, keep)
    h = ctypes.c_void_p()
    if window is None:
        _check(plain(ctypes.byref(d), ctypes.byref(h)))
    else:
        _check(windowed(ctypes.byref(d), _count(window), _count(sinks), ctypes.byref(h)))
    return Plan(h.value, batch)


def ca_plan_host(batch, window=None, sinks=0) -> Plan:
    """Validate `batch` and build its launch schedule on the host only (no GPU needed).  With a window a row sees, of the keys up to
    its own position p, those with p - j < window or j < sinks (ca_plan_window of the header); without one, `sinks` has no effect."""
    return _planned(batch, window, sinks, lib().ca_plan_host, lib().ca_plan_window_host)


def ca_plan(batch, window=None, sinks=0) -> Plan:
    """ca_plan_host + upload of the schedule to the current device."""
    return _planned(batch, window, sinks, lib().ca_plan, lib().ca_plan_window)


def _stream_ptr(stream):
    """The hipStream_t as an integer (or None): torch's current stream unless one is given."""
    if stream is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None and torch.cuda.is_initialized():  # the handle without a Stream object around it: 0.4 us, not 3.7
            return raw(torch.cuda.current_device()) or None
        return torch.cuda.current_stream().cuda_stream or None if torch.cuda.is_available() else None
    return (stream if isinstance(stream, int) else stream.cuda_stream) or None


def _p(t):
    return t.data_ptr() if t is not None and t.numel() > 0 else None


def _expect(t, shape, dtype, name):
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name}: expected contiguous device tensor {tuple(shape)} {dtype}, got {tuple(t.shape)} {t.dtype}")


def ca_forward(plan: Plan, q, k, v, o, lse, ws=None, stream=None):
    """Launch the fused forward on torch's current stream (or `stream`).  Writes o (bf16) and lse (fp32), and, if it has room
    for the partial results of cut units, ws: calls that may overlap in time need one each, or none."""
    import torch
    b, bf16 = plan.batch, torch.bfloat16
    qs, ks = (b.total_q, b.n_q_heads, b.head_dim), (b.total_kv, b.n_kv_heads, b.head_dim)
    _expect(q, qs, bf16, "q")
    _expect(k, ks, bf16, "k")
    _expect(v, ks, bf16, "v")
    _expect(o, qs, bf16, "o")
    _expect(lse, (b.n_q_heads, b.total_q), torch.float32, "lse")
    wsb = ws.numel() * ws.element_size() if ws is not None else 0
    _check(lib().ca_forward(plan.handle, _p(q), _p(k), _p(v), _p(o), _p(lse), _p(ws), wsb, _stream_ptr(stream)))


def _expect_backward(b, q, k, v, o, d_o, lse, dq, dk, dv):
    import torch
    bf16 = torch.bfloat16
    qs, ks = (b.total_q, b.n_q_heads, b.head_dim), (b.total_kv, b.n_kv_heads, b.head_dim)
    _expect(q, qs, bf16, "q")
    _expect(o, qs, bf16, "o")
    _expect(d_o, qs, bf16, "d_o")
    _expect(dq, qs, bf16, "dq")
    _expect(k, ks, bf16, "k")
    _expect(v, ks, bf16, "v")
    _expect(dk, ks, bf16, "dk")
    _expect(dv, ks, bf16, "dv")
    _expect(lse, (b.n_q_heads, b.total_q), torch.float32, "lse")


def ca_backward(plan: Plan, q, k, v, o, d_o, lse, dq, dk, dv, ws, stream=None):
    """Launch the backward on torch's current stream (or `stream`).  Writes dq, dk, dv (bf16)."""
    _expect_backward(plan.batch, q, k, v, o, d_o, lse, dq, dk, dv)
    wsb = ws.numel() * ws.element_size() if ws is not None else 0
    _check(lib().ca_backward(plan.handle, _p(q), _p(k), _p(v), _p(o), _p(d_o), _p(lse), _p(dq), _p(dk), _p(dv),
                             _p(ws), wsb, _stream_ptr(stream)))


def ca_backward_static_ws(plan: Plan, q, k, v, o, d_o, lse, dq, dk, dv, stream=None):
    """ca_backward on the library's own device-resident workspace (for callers that may not allocate)."""
    _expect_backward(plan.batch, q, k, v, o, d_o, lse, dq, dk, dv)
    _check(lib().ca_backward_static_ws(plan.handle, _p(q), _p(k), _p(v), _p(o), _p(d_o), _p(lse), _p(dq), _p(dk),
                                       _p(dv), _stream_ptr(stream)))


def _scratch(preferred, needed, device):
    """A uint8 buffer of `preferred` bytes, or of `needed` (None for 0) where the device has no room for that: partial results
    of cut units may take 256 MiB, and a batch that fits without them must go on fitting."""
    import torch
    if preferred > needed:
        try:
            return torch.empty(preferred, dtype=torch.uint8, device=device)
        except torch.cuda.OutOfMemoryError:
            pass
    return torch.empty(needed, dtype=torch.uint8, device=device) if needed else None


def _room_for_sums(n_bytes, device):
    """Whether n_bytes are at most an eighth of the device memory that nobody holds."""
    import torch
    if torch.device(device).type != "cuda" or torch.cuda.is_current_stream_capturing():
        return True
    free = torch.cuda.mem_get_info(device)[0]
    if n_bytes > free // 8:  # what torch's cache holds is free too, but asking for it takes 0.1 ms
        free += torch.cuda.memory_reserved(device) - torch.cuda.memory_allocated(device)
    return n_bytes <= free // 8


def alloc_workspace(plan: Plan, device="cuda", one_pass=None):
    """A torch uint8 buffer big enough for both calls, with room for the partial results of units cut into pieces, or for a
    backward in one pass (torch's allocator returns 256-byte aligned blocks).  The one pass about doubles the buffer: one_pass says
    whether it may; by default where what it adds is at most an eighth of the device memory that is free, so that what the
    program allocates later goes on fitting.  Where the device has no room for the larger buffer it is the smaller one.  Both calls
    write to it: calls that may overlap in time need one each."""
    import torch
    needed, split = max(*plan.workspace_bytes(), 256), max(*plan.workspace_bytes_split(), 256)
    sums = plan.workspace_bytes_one_pass() if one_pass is None or one_pass else 0
    if sums and (one_pass or _room_for_sums(sums - needed, device)):
        try:
            return torch.empty(max(sums, split), dtype=torch.uint8, device=device)
        except torch.cuda.OutOfMemoryError:
            pass
    return _scratch(split, needed, device)


def ca_merge_partials(part_rows, o_part, lse_part, o, lse, o_back=None, lse_back=None, stream=None):
    """Merge partial results over disjoint key windows.  part_rows: device int32 [n_parts, n_rows]; o_part bf16
    [total_q_part, Hq, D], lse_part fp32 [Hq, total_q_part]; writes o bf16 [n_rows, Hq, D] and lse fp32 [Hq, n_rows];
    o_back / lse_back (may be o_part / lse_part) receive the merged values in every partial row."""
    import torch
    n_parts, n_rows = part_rows.shape
    tq, hq, d = o_part.shape
    _expect(part_rows, (n_parts, n_rows), torch.int32, "part_rows")
    _expect(o_part, (tq, hq, d), torch.bfloat16, "o_part")
    _expect(lse_part, (hq, tq), torch.float32, "lse_part")
    _expect(o, (n_rows, hq, d), torch.bfloat16, "o")
    _expect(lse, (hq, n_rows), torch.float32, "lse")
    if o_back is not None:
        _expect(o_back, (tq, hq, d), torch.bfloat16, "o_back")
    if lse_back is not None:
        _expect(lse_back, (hq, tq), torch.float32, "lse_back")
    _check(lib().ca_merge_partials(_p(part_rows), n_rows, n_parts, _p(o_part), _p(lse_part), tq, _p(o), _p(lse),
                                   _p(o_back), _p(lse_back), hq, d, _stream_ptr(stream)))


def ca_sum_partial_dq(part_rows, dq_part, dq, stream=None):
    """dq[r] = sum of the partial query gradients of row r (arguments as in ca_merge_partials)."""
    import torch
    n_parts, n_rows = part_rows.shape
    tq, hq, d = dq_part.shape
    _expect(part_rows, (n_parts, n_rows), torch.int32, "part_rows")
    _expect(dq_part, (tq, hq, d), torch.bfloat16, "dq_part")
    _expect(dq, (n_rows, hq, d), torch.bfloat16, "dq")
    _check(lib().ca_sum_partial_dq(_p(part_rows), n_rows, n_parts, _p(dq_part), tq, _p(dq), hq, d, _stream_ptr(stream)))


# The calls on a cache run once per layer and token: what they check of their tensors is a good part of what the small ones take.
def _on_cache(cache, t, shape, dtype, name) -> int:
    """Address of a contiguous tensor of that shape and type on the cache's device."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != cache.index or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous tensor {tuple(shape)} {dtype} on {cache.device}, got {tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


def _cache_batch(cache, rows, q_start, kv_len, page_table) -> CacheBatch:
    i32, n = cache.i32, kv_len.shape[0]
    if page_table.dim() != 2:
        raise ValueError(f"page_table: expected [{n}, pages], got {tuple(page_table.shape)}")
    width = page_table.shape[1]
    return CacheBatch(n, width, rows, _on_cache(cache, q_start, (n + 1,), i32, "q_start"), _on_cache(cache, kv_len, (n,), i32, "kv_len"),
                      _on_cache(cache, page_table, (n, width), i32, "page_table"))


def _cache_stream(cache, stream):
    """The stream's address; the cache's memory has to be on the current device, whose streams order the work on it."""
    current = cache.current_device()
    if cache.index != current:
        raise ValueError(f"the cache is on {cache.device}, the current device is {current}")
    return _stream_ptr(stream) if stream is not None or cache.raw_stream is None else cache.raw_stream(current)


def ca_cache_append(cache, k, v, q_start, kv_len, page_table, stream=None):
    """Quantise the rows of k and v (bf16 [rows, n_kv_heads, head_dim]) into the pages of their sequences (cache: cache.KVCache; the
    arrays: device int32, see the header).  On torch's current stream, or `stream`."""
    rows = k.shape[0]
    shape = (rows, cache.n_kv_heads, cache.head_dim)
    kp, vp = _on_cache(cache, k, shape, cache.bf16, "k"), _on_cache(cache, v, shape, cache.bf16, "v")
    b = _cache_batch(cache, rows, q_start, kv_len, page_table)
    _check(lib().ca_cache_append(cache.desc_ref, ctypes.byref(b), kp, vp, _cache_stream(cache, stream)))


def ca_cache_attend(cache, q, o, lse, q_start, kv_len, page_table, ws, window=None, sinks=0, softmax_scale=0.0, stream=None):
    """Attention of the rows of q (bf16 [rows, n_q_heads, head_dim]) over the cached tokens of their sequences.  Writes o (like q) and,
    unless it is None, lse (fp32 [n_q_heads, rows]); ws: alloc_cache_workspace."""
    rows, hq, _ = shape = q.shape
    if window is None:
        window = 0
    elif operator.index(window) < 1:
        raise ValueError(f"window {window}: at least 1, or None")
    qp = _on_cache(cache, q, (rows, hq, cache.head_dim), cache.bf16, "q")
    op = _on_cache(cache, o, shape, cache.bf16, "o")
    lp = None if lse is None else _on_cache(cache, lse, (hq, rows), cache.f32, "lse")
    b = _cache_batch(cache, rows, q_start, kv_len, page_table)
    wp, n = (None, 0) if ws is None else (_on_cache(cache, ws, ws.shape, ws.dtype, "ws"), ws.numel() * ws.element_size())
    _check(lib().ca_cache_attend(cache.desc_ref, ctypes.byref(b), hq, softmax_scale, _count(window), _count(sinks), qp, op, lp, wp,
                                 n, _cache_stream(cache, stream)))


def ca_cache_attend_shared(cache, q, o, lse, q_start, kv_len, page_table, group_start, prefix_pages, ws, softmax_scale=0.0, stream=None):
    """ca_cache_attend where groups of sequences share their first pages, which are attended once for all rows of a group: group g has the sequences
    group_start[g] .. group_start[g + 1] - 1, and their first prefix_pages[g] pages are the same (device int32; cache.Sequences.groups, which says when it pays).
    ws: alloc_shared_workspace."""
    rows, hq, _ = shape = q.shape
    qp = _on_cache(cache, q, (rows, hq, cache.head_dim), cache.bf16, "q")
    op = _on_cache(cache, o, shape, cache.bf16, "o")
    lp = None if lse is None else _on_cache(cache, lse, (hq, rows), cache.f32, "lse")
    b = _cache_batch(cache, rows, q_start, kv_len, page_table)
    n = prefix_pages.shape[0]
    g = CacheGroups(n, _on_cache(cache, group_start, (n + 1,), cache.i32, "group_start"), _on_cache(cache, prefix_pages, (n,), cache.i32, "prefix_pages"))
    wp, wn = (None, 0) if ws is None else (_on_cache(cache, ws, ws.shape, ws.dtype, "ws"), ws.numel() * ws.element_size())
    _check(lib().ca_cache_attend_shared(cache.desc_ref, ctypes.byref(b), ctypes.byref(g), hq, softmax_scale, qp, op, lp, wp, wn,
                                        _cache_stream(cache, stream)))


def alloc_shared_workspace(cache, n_q_heads, rows, device=None):
    """A torch uint8 buffer big enough for ca_cache_attend_shared on that cache with up to that many rows.  Calls that may overlap in time need one
    each."""
    import torch
    n = ctypes.c_size_t()
    _check(lib().ca_cache_attend_shared_workspace_bytes(cache.desc_ref, operator.index(n_q_heads), operator.index(rows), ctypes.byref(n)))
    return torch.empty(n.value, dtype=torch.uint8, device=cache.device if device is None else device)


def ca_cache_read(cache, k, v, q_start, kv_len, page_table, stream=None):
    """The rows of the batch out of the cache: k and v (bf16 [rows, n_kv_heads, head_dim]; one of them may be None) are written."""
    if k is None and v is None:
        raise ValueError("k and v: one of them at least")
    rows = (v if k is None else k).shape[0]
    shape = (rows, cache.n_kv_heads, cache.head_dim)
    kp, vp = (None if x is None else _on_cache(cache, x, shape, cache.bf16, name) for x, name in ((k, "k"), (v, "v")))
    b = _cache_batch(cache, rows, q_start, kv_len, page_table)
    _check(lib().ca_cache_read(cache.desc_ref, ctypes.byref(b), kp, vp, _cache_stream(cache, stream)))


def ca_cache_copy_pages(cache, src, dst, stream=None):
    """Copy page src[i] of the cache to page dst[i] (device int32 [n]; no page is written twice or both written and read)."""
    n = src.shape[0]
    sp, dp = _on_cache(cache, src, (n,), cache.i32, "src"), _on_cache(cache, dst, (n,), cache.i32, "dst")
    _check(lib().ca_cache_copy_pages(cache.desc_ref, sp, dp, n, _cache_stream(cache, stream)))


def alloc_cache_workspace(cache, n_q_heads, device=None):
    """A torch uint8 buffer big enough for ca_cache_attend on that cache.  Calls that may overlap in time need one each."""
    import torch
    n = ctypes.c_size_t()
    _check(lib().ca_cache_attend_workspace_bytes(cache.desc_ref, operator.index(n_q_heads), ctypes.byref(n)))
    return torch.empty(n.value, dtype=torch.uint8, device=cache.device if device is None else device)


def rows_in_line(t):
    """t [rows, heads, head_dim] itself where its rows are 16-byte aligned and each of them is one run of memory, otherwise a copy."""
    import torch
    rows, heads, d = t.shape
    s = t.stride()
    if s[2] == 1 and (heads == 1 or s[1] == d) and (rows == 1 or (s[0] % 8 == 0 and s[0] >= heads * d)) and t.data_ptr() % 16 == 0:
        return t
    return t.clone(memory_format=torch.contiguous_format)


def _rows(rotation, t, shape, name):
    """Address and row stride of a bf16 tensor [rows, heads, head_dim] on the rotation's device, each of whose rows is one run of memory."""
    if t.dtype is rotation.bf16 and t.shape == shape and t.get_device() == rotation.index:
        rows, heads, d = shape
        if t.is_contiguous():
            return t.data_ptr(), heads * d
        s = t.stride()
        if s[2] == 1 and (heads == 1 or s[1] == d) and (rows == 1 or (s[0] >= heads * d and s[0] % 8 == 0)):
            return t.data_ptr(), s[0] if rows > 1 else heads * d
    raise ValueError(f"{name}: expected bf16 tensor {tuple(shape)} on {rotation.device}, whose rows are runs of memory a multiple of 8 elements apart, "
                     f"got {tuple(t.shape)} {t.dtype} on {t.device} with strides {t.stride()}")


def _line(rotation, t, shape, dtype, name):
    if t.dtype is not dtype or t.shape != shape or t.get_device() != rotation.index or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous tensor {tuple(shape)} {dtype} on {rotation.device}, got {tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


# Descriptions as packed bytes, which take a third of the time of a ctypes.Structure (these calls run once per layer and token too).
_ROTATE_TENSOR = struct.Struct("=6Q4q2i")  # ca_rotate_tensor
_ROTATE_WHERE = struct.Struct("=iiq3Q")     # ca_cache_batch


def _rotate_tensor(rotation, x, dy, y, pos, where, gain, dgain, name, gaps=0):
    """A ca_rotate_tensor; x None: of a gradient without a gain."""
    if y is None:
        raise ValueError(f"{name}: the result is None")
    shape = y.shape
    if len(shape) != 3 or shape[2] != rotation.head_dim:
        raise ValueError(f"{name}: expected [rows, heads, {rotation.head_dim}], got {tuple(shape)}")
    xp = xs = dp = ds = gp = dgp = pp = 0
    yp, ys = _rows(rotation, y, shape, name)
    if x is not None:
        xp, xs = _rows(rotation, x, shape, name)
    if dy is not None:
        dp, ds = _rows(rotation, dy, shape, name)
    if gain is not None:
        gp = _line(rotation, gain, shape[2:], rotation.f32, name)
        if dy is not None:
            dgp = _line(rotation, dgain, shape[2:], rotation.f32, name)
    if where is None:
        if pos is None:
            raise ValueError(f"{name}: neither positions nor sequences are given")
        pp = _line(rotation, pos, shape[:1], rotation.i32, name)
    return _ROTATE_TENSOR.pack(xp, dp, yp, gp, dgp, pp, shape[0], xs, ds, ys, shape[1], gaps)


def _rotate_where(rotation, where, rows):
    """The sequences as a ca_cache_batch, or None."""
    if where is None:
        return None
    start, lens = where[0], where[1]
    n = lens.shape[0]
    return _ROTATE_WHERE.pack(n, 0, rows, _line(rotation, start, (n + 1,), rotation.i32, "q_start"), _line(rotation, lens, (n,), rotation.i32, "kv_len"), 0)


def _rotate_stream(rotation, stream):
    """The stream's address; the tensors have to be on the current device, whose streams order the work on it."""
    current = rotation.current_device()
    if rotation.index != current:
        raise ValueError(f"the rotation is on {rotation.device}, the current device is {current}")
    return _stream_ptr(stream) if stream is not None or rotation.raw_stream is None else rotation.raw_stream(current)


def ca_rotate(rotation, q, k, q_out, k_out, q_pos=None, k_pos=None, where=None, q_gain=None, k_gain=None, eps=1e-6, stream=None):
    """Norm (with a gain) and turn of the rows of q, and of k unless it is None, in one launch on torch's current stream, or `stream`
    (rotation: rotary.Rotation).  q, k and the outputs: bf16 [rows, heads, head_dim], each row a run of memory, so that views of a joint projection
    will do; an output may be its input.  Positions: q_pos and k_pos (device int32 [rows]; k_pos None: those of q), or where = (q_start, kv_len, ..) of
    the sequences of a call on a cache: rows are their last ones, and rows of no sequence are left as they are.  Gains: fp32 [head_dim]."""
    n, tensors = 1, _rotate_tensor(rotation, q, None, q_out, q_pos, where, q_gain, None, "q, its output, positions or gain")
    if k is None:
        if k_out is not None or k_gain is not None:
            raise ValueError("an output or a gain of k without k")
    else:
        n, tensors = 2, tensors + _rotate_tensor(rotation, k, None, k_out, q_pos if k_pos is None else k_pos, where, k_gain, None,
                                                 "k, its output, positions or gain")
    _check(lib().ca_rotate(rotation.desc_ref, tensors, n, _rotate_where(rotation, where, q.shape[0]), eps, _rotate_stream(rotation, stream)))


def ca_rotate_backward(rotation, q, k, dq_out, dk_out, dq, dk, q_pos=None, k_pos=None, where=None, q_gain=None, k_gain=None, dq_gain=None,
                       dk_gain=None, eps=1e-6, ws=None, stream=None, q_gaps=False, k_gaps=False):
    """Gradients of ca_rotate: dq and dk (may be dq_out and dk_out) and, with gains, dq_gain and dk_gain (fp32 [head_dim]), from dq_out and dk_out
    (dk_out None: of q alone).  q and k are needed where there is a gain, as is ws (alloc_rotate_workspace).  q_gaps, k_gaps: rows at
    position rotary.GAP take no part, whatever they hold: their dq (dk) is left as it is, and the gain's gradient has nothing of them."""
    n, tensors, rows = 0, b"", 0
    for x, dy, dx, pos, gain, dgain, gaps, name in ((q, dq_out, dq, q_pos, q_gain, dq_gain, q_gaps, "q"),
                                                    (k, dk_out, dk, q_pos if k_pos is None else k_pos, k_gain, dk_gain, k_gaps, "k")):
        if dy is None:
            if dx is not None or dgain is not None:
                raise ValueError(f"{name}: a gradient without that of the output")
            continue
        if gain is not None and (x is None or dgain is None):
            raise ValueError(f"{name}: with a gain the gradient needs the input, and a tensor for that of the gain")
        tensors += _rotate_tensor(rotation, x if gain is not None else None, dy, dx, pos, where, gain, dgain, f"{name}, its gradients, positions or gain", gaps)
        n, rows = n + 1, dy.shape[0]
    if n == 0:
        raise ValueError("neither dq_out nor dk_out")
    wp, wn = (None, 0) if ws is None else (_line(rotation, ws, ws.shape, ws.dtype, "ws"), ws.numel() * ws.element_size())
    _check(lib().ca_rotate_backward(rotation.desc_ref, tensors, n, _rotate_where(rotation, where, rows), eps, wp, wn, _rotate_stream(rotation, stream)))


def alloc_rotate_workspace(device="cuda"):
    """A torch uint8 buffer big enough for ca_rotate_backward.  Calls that may overlap in time need one each."""
    import torch
    return torch.empty(lib().ca_rotate_backward_workspace_bytes(), dtype=torch.uint8, device=device)


def ca_mfma_stream(operands, n_mfma_per_wave, sums, side_work=0, stream=None, shape=32):
    """Back-to-back bf16 MFMAs from registers in sums.shape[0] workgroups (a calibration aid; see the header); shape 32: 32x32x16,
    16: 16x16x32 (ca_mfma_stream16)."""
    import torch
    _expect(operands, (16, 256, 8), torch.bfloat16, "operands")
    n_wg = sums.shape[0]
    _expect(sums, (n_wg, 256), torch.float32, "sums")
    if shape not in (16, 32):
        raise ValueError(f"shape {shape}: 16 or 32")
    stream_of = lib().ca_mfma_stream if shape == 32 else lib().ca_mfma_stream16
    _check(stream_of(_p(operands), int(n_mfma_per_wave), n_wg, int(side_work), _p(sums), _stream_ptr(stream)))


def ca_xcd_map(n_workgroups, threads_per_workgroup=256, device="cuda", stream=None):
    """XCD id of every workgroup of a launch of that shape (int32 tensor on the device)."""
    import torch
    out = torch.full((n_workgroups,), -1, dtype=torch.int32, device=device)
    _check(lib().ca_xcd_map(int(n_workgroups), int(threads_per_workgroup), _p(out), _stream_ptr(stream)))
    return out


def ca_atomic_stream(operands, tiles, n_workgroups, steps, mfma_per_step, atomics_per_step, sums, stream=None):
    """fp32 atomic adds into 32 KiB tiles next to an MFMA stream (a calibration aid; see the header)."""
    import torch
    _expect(operands, (16, 256, 8), torch.bfloat16, "operands")
    n_tiles = tiles.shape[1]
    _expect(tiles, (8, n_tiles, 8192), torch.float32, "tiles")
    _expect(sums, (n_workgroups, 256), torch.float32, "sums")
    _check(lib().ca_atomic_stream(_p(operands), _p(tiles), int(n_tiles), int(n_workgroups), int(steps),
                                  int(mfma_per_step), int(atomics_per_step), _p(sums), _stream_ptr(stream)))
