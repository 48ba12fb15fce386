"""Appending to pages whose scales are no powers of two (a cache that something else has filled), bit for bit: the scale becomes the smallest power of two that holds
the new tokens and is no less than it was, and what the page held is rounded again."""
import numpy as np
import pytest
import torch

import cache_util as U
from paper_2510_18121_amd import binding as B
from paper_2510_18121_amd.cache import KVCache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int32), device=DEV)


def power_up(x):
    """The smallest power of two that is at least x > 0."""
    m, e = np.frexp(x)
    return np.ldexp(1.0, np.where(m == 0.5, e - 1, e))


@pytest.mark.parametrize("heads,d", [(3, 64), (2, 128)])
@pytest.mark.parametrize("rows", [1, 3, 4, 33, 70])
@pytest.mark.parametrize("size", [2.0 ** -9, 1.0, 37.0])
def test_append_to_scales_of_any_value(heads, d, rows, size):
    """New tokens smaller than, as large as and larger than what the pages hold; from the first, an inner and the last token of a page on."""
    held_before = [0, 1, 6, 63, 100, 128]
    lens = [x + rows for x in held_before]
    table, pages = U.layout(lens, seed=51)
    g = torch.Generator(device=DEV).manual_seed(52)
    c = KVCache.empty(pages, heads, d, DEV)
    for codes, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
        scale.copy_(torch.rand(scale.shape, generator=g, device=DEV) * 0.02 + 1e-3)
        codes.copy_((torch.randn(codes.shape, generator=g, device=DEV) * 100).clamp(-448, 448).to(U.F8))
    new = (torch.randn(2, rows * len(lens), heads, d, generator=g, device=DEV) * size).to(torch.bfloat16)
    want = {"k": c.k.cpu().double().numpy(), "v": c.v.cpu().double().numpy().transpose(0, 1, 3, 2).copy(), "ks": c.k_scale.cpu().double().numpy(),
            "vs": c.v_scale.cpu().double().numpy()}
    fresh, row = new.double().cpu().numpy(), 0
    for i, total in enumerate(lens):
        p = total - rows
        while p < total:
            page, a = table[i, p // 64], p % 64
            e = min(64, a + total - p)
            for x, codes, scale in ((fresh[0], want["k"][page], want["ks"][page]), (fresh[1], want["v"][page], want["vs"][page])):
                x = x[row:row + e - a].transpose(1, 0, 2)
                now = np.maximum(power_up(np.abs(x).max((1, 2)) / 448), 2.0 ** -126)
                if a > 0:
                    now = np.maximum(now, power_up(scale))
                    again = codes * (scale / now)[:, None, None]
                    # (the kernel's product is one of fp32, off by 2^-24: none of these may lie as near to a tie)
                    assert all((U.round_e4m3(again * f) == U.round_e4m3(again)).all() for f in (1 - 2.0 ** -22, 1 + 2.0 ** -22))
                    codes[:] = U.round_e4m3(again)
                codes[:, a:e] = U.round_e4m3(x / now[:, None, None])
                scale[:] = now
            row, p = row + e - a, p + e - a
    B.ca_cache_append(c, new[0], new[1], i32(np.arange(len(lens) + 1) * rows), i32(lens), i32(table))
    got = {"k": c.k.cpu().double().numpy(), "v": c.v.cpu().double().numpy().transpose(0, 1, 3, 2), "ks": c.k_scale.cpu().double().numpy(),
           "vs": c.v_scale.cpu().double().numpy()}
    for name in want:
        assert np.array_equal(got[name], want[name]), name
