"""Where the kernels hold P in two bf16 operands, O is as exact as that: attention over the cache with up to 32 rows a tile, and the windowed
forward's rows whose context ends in the first tile of keys."""
import numpy as np
import pytest
import torch

import accuracy_util as A
import cache_util as C
import window_util as U
from paper_2510_18121_amd import binding as B
from paper_2510_18121_amd import workloads as W
from paper_2510_18121_amd.cache import KVCache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int32), device=DEV)


def check_cache(hq, hkv, d, n, lens, window=None, sinks=0):
    table, pages = C.layout(lens, seed=41)
    g = torch.Generator(device=DEV).manual_seed(42)
    c = KVCache.empty(pages, hkv, d, DEV)
    for codes, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
        x = torch.randn(codes.shape, generator=g, device=DEV)
        scale.copy_(x.abs().amax((2, 3)) / 448 * 1.1)
        codes.copy_((x / scale[:, :, None, None]).to(C.F8))
    q = torch.randn(sum(n), hq, d, generator=g, device=DEV).to(torch.bfloat16)
    o, ws = torch.empty_like(q), B.alloc_cache_workspace(c, hq)
    B.ca_cache_attend(c, q, o, None, i32(np.concatenate([[0], np.cumsum(n)])), i32(lens), i32(table), ws, window=window, sinks=sinks)
    k, v = C.values(c.k, c.k_scale), C.values(c.v, c.v_scale).transpose(2, 3)
    for rows, h, a, p, v_of, want in A.cache_rows(k, v, q, n, lens, table, window, sinks):
        A.check(o[rows, h], want, A.row_bound(a, p, v_of, want))


LENS = [1, 2, 3, 5, 9, 17, 33, 64, 65, 130]


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (8, 1, 128), (3, 3, 128), (16, 1, 64)])
@pytest.mark.parametrize("rows", [1, 2])
def test_few_keys(hq, hkv, d, rows):
    check_cache(hq, hkv, d, [min(rows, x) for x in LENS], LENS)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (8, 2, 128), (16, 2, 64), (16, 2, 128)])
@pytest.mark.parametrize("length,seqs", [(300, 6), (2300, 6), (150, 260)])
def test_short_windows_of_long_contexts(hq, hkv, d, length, seqs):
    """Tiles of 16 and of 32 rows; two, four and eight waves to a workgroup."""
    lens = [length - i % 70 for i in range(seqs)]
    check_cache(hq, hkv, d, [4] * seqs, lens, window=5, sinks=2)


@pytest.mark.parametrize("heads,d", [((4, 2), 64), ((4, 1), 128), ((3, 3), 128), ((8, 1), 64)])
@pytest.mark.parametrize("window,sinks", [(1, 3), (7, 0), (40, 2), (100, 0)])
def test_windowed_rows_of_the_first_tile(heads, d, window, sinks):
    lens = [64, 30, 200, 64, 101]
    b = W.custom(lens, [(i, 0, x) for i, x in enumerate(lens)], *heads, d, seed=43)
    q, k, v, _ = W.make_tensors(b, DEV)
    plan = B.ca_plan(b, window=window, sinks=sinks)
    o, lse = torch.empty_like(q), torch.empty(heads[0], b.total_q, device=DEV)
    B.ca_forward(plan, q, k, v, o, lse, None)
    see = torch.from_numpy(U.visible(b, window, sinks))
    qd, kd, vd = (x.double().cpu() for x in (q, k, v))
    first = np.concatenate([np.arange(s, s + min(n, 64)) for s, n in zip(np.cumsum([0] + lens[:-1]), lens)])
    for h in range(heads[0]):
        kh, vh, qh = kd[:, h * heads[1] // heads[0]], vd[:, h * heads[1] // heads[0]], qd[first, h]
        s = (qh @ kh.T * d ** -0.5).masked_fill(~see[first], -np.inf)
        p = torch.softmax(s, 1)
        want = p @ vh
        A.check(o[first, h], want, A.row_bound(qh.abs() @ kh.abs().T * d ** -0.5, p, vh, want))
