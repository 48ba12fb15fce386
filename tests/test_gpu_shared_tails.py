"""Tails of several rows each, as many bytes as the last cache holds and more, against attention without sharing."""
import pytest
import torch

import numpy as np

from paper_2510_18121_amd import binding as B
from test_gpu_cache import DEV, filled, i32, queries
from test_gpu_cache_shared import attend, layout

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 4, 5, 8])
@pytest.mark.parametrize("tail", [5000, 7500])
def test_tails_of_one_tile_and_of_two(rows, tail):
    """4 to 32 rows per KV head.  Each call is off by at most 2^-8 of O and 2^-13 of what the probabilities and values weigh (P in two operands, sums and
    exponentials), which over thousands of values of unlike signs is some 2^6 times O's norm at the most, so that by 2 (2^-8 + 2^-7) of O the two differ at most."""
    tails, d = [tail + 37 * i for i in range(24)], 128
    lens = [64 * 20 + t for t in tails]
    table, pages = layout([(24, 20)], lens)
    c, n = filled(pages, 8, d), [rows] * 24
    q = queries(sum(n), 32, d)
    o, lse = attend(c, q, n, lens, table, [(24, 20)])
    want, want_lse = torch.empty_like(q), torch.empty_like(lse)
    B.ca_cache_attend(c, q, want, want_lse, i32(np.concatenate([[0], np.cumsum(n)])), i32(lens), i32(table), B.alloc_cache_workspace(c, 32))
    assert (o.double() - want.double()).norm() <= (2.0 ** -7 + 2.0 ** -6) * want.double().norm()
    assert (lse - want_lse).abs().max() <= 2e-4
