"""Attention of groups holds P in two bf16 operands where ca_cache_attend does, of the shared keys too, whatever the groups' sizes and whoever else is in
the call."""
import pytest
import torch

import accuracy_util as A
import cache_util as C
import shared_accuracy_util as S
from paper_2510_18121_amd.cache import KVCache
from test_gpu_cache_shared import attend, layout

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def check(hq, hkv, d, groups, n, tails, far=False):
    prefix = [p for m, p in groups for _ in range(m)]
    lens = [64 * p + t for p, t in zip(prefix, tails)]
    table, pages = layout(groups, lens, seed=51)
    g = torch.Generator(device=DEV).manual_seed(52)
    c = KVCache.empty(pages, hkv, d, DEV)
    for codes, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
        x = torch.randn(codes.shape, generator=g, device=DEV)
        scale.copy_(x.abs().amax((2, 3)) / 448 * 1.1)
        codes.copy_((x / scale[:, :, None, None]).to(C.F8))
    if far:  # scales that the exponent does not take
        c.v_scale *= 2.0 ** 45
        c.v_scale[torch.as_tensor(table[0, :1], device=DEV).long()] *= 2.0 ** -5
    q = (0.1 * torch.randn(sum(n), hq, d, generator=g, device=DEV)).to(torch.bfloat16)
    o, _ = attend(c, q, n, lens, table, groups, lse=False)
    k, v = C.values(c.k, c.k_scale), C.values(c.v, c.v_scale).transpose(2, 3)
    for rows, h, a, p, v_of, want in A.cache_rows(k, v, q, n, lens, table, None, 0):
        A.check(o[rows, h], want, S.bound(a, p, v_of, want))


HEADS = [(8, 2, 64), (16, 4, 128), (3, 3, 128), (16, 1, 64)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("members,shared", [(2, 1), (36, 1), (36, 2), (40, 6)])
def test_answers_to_one_prompt(hq, hkv, d, members, shared):
    """Prefixes in tiles of 16 and of 128 rows, whole and cut."""
    check(hq, hkv, d, [(members, shared)], [1] * members, [1 + 7 * i % 301 for i in range(members)])


@pytest.mark.parametrize("hq,hkv,d", HEADS[:2])
def test_drafts_of_several_rows(hq, hkv, d):
    check(hq, hkv, d, [(12, 2), (9, 1)], [1 + i % 6 for i in range(21)], [6 + 11 * i for i in range(21)])


@pytest.mark.parametrize("members", [40, 2])
def test_sequences_that_share_nothing_in_the_call(members):
    """As many groups of no pages, so that the average group is small, or one that is not."""
    check(8, 2, 128, [(members, 2)] + [(1, 0)] * 60, [1] * (members + 60), [1 + 5 * i % 290 for i in range(members + 60)])
    check(8, 2, 128, [(members, 2), (60, 0)], [1] * (members + 60), [1 + 5 * i % 290 for i in range(members + 60)])


def test_scales_that_the_exponent_does_not_take():
    check(8, 2, 64, [(20, 2)], [1] * 20, [10 + i for i in range(20)], far=True)
    check(8, 2, 128, [(20, 5)], [1] * 20, [10 + i for i in range(20)], far=True)
