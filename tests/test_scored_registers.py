"""Spilled vector registers of the kernels for scored attention, weights and eviction, read from the metadata of the built library."""
import os

import pytest

from paper_2403_20137_amd import kvbfp

kernels = pytest.importorskip("test_kernel_registers").kernels
SPILLS = {"scored_splitILi8ELb1ELi1ELi16E": 3, "scored_splitILi8ELb1ELi1ELi8E": 1}       # stated beside the code


@pytest.mark.skipif(not os.path.exists(kvbfp.LIB_PATH), reason="library not built")
def test_nothing_else_spills():
    got = {n: k[".vgpr_spill_count"] for n, k in kernels().items() if any(x in n for x in ("scored_", "accumulate_weights", "evict_"))}
    assert len(got) == 24 + 28 + 12 + 24 + 12 + 3, len(got)
    for name, count in got.items():
        allowed = next((v for k, v in SPILLS.items() if k in name), 0)
        assert count <= allowed, (name, count)
