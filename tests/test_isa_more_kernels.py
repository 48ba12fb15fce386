"""Static checks of the generated assembly of the rotation's kernels, of reading the cache and of attention of groups (no GPU): nothing is spilled to
memory, no vector instruction is inline assembly, and what a transcendental instruction gives is not read too early."""
import os

import pytest

from paper_2510_18121_amd import isa_check as C

pytestmark = pytest.mark.skipif(not os.path.exists(os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")),
                                reason="hipcc is needed to produce the assembly")


@pytest.mark.parametrize("source,kernels,transcendental", [
    ("ca_rotate.hip", {"ca_rotate_kernel": 24, "ca_rotate_gain_kernel": 2}, 20),
    ("ca_cache_read.hip", {"ca_cache_read_kernel": 4}, 0),
    ("ca_cache_shared.hip", {"ca_cache_shared_kernel": 6, "ca_cache_join_kernel": 6}, 50)])
def test_kernels_keep_everything_in_registers(source, kernels, transcendental):
    asm = C.compile_to_asm(source)
    for name, n in kernels.items():
        bodies = C.kernel_bodies(asm, name)
        assert len(bodies) == n, name
        assert not any("scratch_" in body for body in bodies), name
    assert C.assembly_vector_instructions(asm) == []
    n, bad = C.check_trans_use(asm)
    assert n >= transcendental and not bad, bad
