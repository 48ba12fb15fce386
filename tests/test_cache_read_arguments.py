"""What reading a cache back refuses, without a GPU."""
import ctypes

import pytest

from paper_2510_18121_amd import binding as B
from paper_2510_18121_amd.cache import CacheDesc

PTR = 1 << 20


def call(cache=None, batch=None, k=PTR, v=PTR):
    c, b = CacheDesc(4, 2, 128, PTR, PTR, PTR, PTR), B.CacheBatch(2, 3, 10, PTR, PTR, PTR)
    for t, fields in ((c, cache), (b, batch)):
        for name, x in (fields or {}).items():
            setattr(t, name, x)
    return B.lib().ca_cache_read(ctypes.byref(c), ctypes.byref(b), k, v, None)


@pytest.mark.parametrize("want,kw", [
    (B.CA_ERR_UNSUPPORTED, {"cache": {"head_dim": 96}}), (B.CA_ERR_INVALID_ARG, {"cache": {"k": None}}), (B.CA_ERR_INVALID_ARG, {"cache": {"v": PTR + 4}}),
    (B.CA_ERR_UNSUPPORTED, {"batch": {"n_seqs": 4097}}), (B.CA_ERR_INVALID_ARG, {"batch": {"kv_len": None}}), (B.CA_ERR_INVALID_ARG, {"batch": {"total_rows": -1}}),
    (B.CA_ERR_INVALID_ARG, {"k": None, "v": None}), (B.CA_ERR_INVALID_ARG, {"k": PTR + 2}), (B.CA_ERR_INVALID_ARG, {"v": PTR + 8}),
    (B.CA_ERR_UNSUPPORTED, {"batch": {"total_rows": (1 << 30) - 1}, "cache": {"n_kv_heads": 1024}})])
def test_calls_that_are_refused(want, kw):
    assert call(**kw) == want
    assert B.lib().ca_last_error()


def test_null_descriptions():
    assert B.lib().ca_cache_read(None, None, PTR, PTR, None) == B.CA_ERR_INVALID_ARG


@pytest.mark.parametrize("batch", [{"n_seqs": 0}, {"total_rows": 0}, {"table_width": 0}])
def test_nothing_to_do_is_no_launch(batch):
    assert call(batch=batch) == B.CA_OK


def test_neither_of_the_two_is_refused():
    with pytest.raises(ValueError):
        B.ca_cache_read(None, None, None, None, None, None)
