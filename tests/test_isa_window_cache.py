"""Static checks of the generated assembly of the windowed and the cache kernels (no GPU): nothing is spilled to memory, and no vector
instruction is inline assembly."""
import os

import pytest

from paper_2510_18121_amd import isa_check as C

pytestmark = pytest.mark.skipif(not os.path.exists(os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")),
                                reason="hipcc is needed to produce the assembly")


@pytest.mark.parametrize("source,kernels", [("ca_window.hip", {"ca_fwd_window_kernel": 2, "ca_bwd_window_kernel": 2, "ca_window_prep_kernel": 2}),
                                            ("ca_cache.hip", {"ca_cache_attend_kernel": 10, "ca_cache_chunk_kernel": 2, "ca_cache_combine_kernel": 6,
                                                              "ca_cache_append_kernel": 2, "ca_cache_copy_kernel": 1})])
def test_kernels_keep_everything_in_registers(source, kernels):
    asm = C.compile_to_asm(source)
    for name, n in kernels.items():
        bodies = C.kernel_bodies(asm, name)
        assert len(bodies) == n, name
        assert not any("scratch_" in body for body in bodies), name
    assert C.assembly_vector_instructions(asm) == []
    n, bad = C.check_trans_use(asm)
    assert n > 50 and not bad, bad
