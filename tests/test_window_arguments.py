"""Windows and sinks of any size, as Python's integers are (no GPU)."""
import pytest

import window_util as U
from paper_2510_18121_amd import binding as B


@pytest.mark.parametrize("far", [(1 << 63) - 1, 1 << 63, (1 << 64) + 5, 10 ** 30])
def test_windows_and_sinks_beyond_64_bits(far):
    """A window that no position reaches hides nothing; sinks beyond every position are all keys; neither is taken modulo 2^64."""
    b = U.batch([300], [(0, 0, 300)], 2, 1, 64)
    plan = B.ca_plan_host(b, window=far, sinks=3)
    assert plan.info() == B.ca_plan_host(b).info() and [x.size for x in plan.window_units()] == [0, 0, 0]
    some, all_of_them = (B.ca_plan_host(b, window=5, sinks=n).window_units() for n in (1 << 20, far))
    assert all((x == y).all() for x, y in zip(some, all_of_them))
    for window, sinks in ((-far, 0), (5, -far)):
        with pytest.raises(B.CaError) as e:
            B.ca_plan_host(b, window=window, sinks=sinks)
        assert e.value.code == B.CA_ERR_INVALID_ARG
