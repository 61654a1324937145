"""Registers of the key-value cache's kernels (CPU; reads this repository's own
library): nothing is spilled, and matrix-core results, which attention reads
after branches, stay out of accumulation registers (this compiler reads those
too early there)."""
import re

import pytest

from test_build_resources import kernels  # noqa: F401  (a fixture)


@pytest.mark.parametrize("name,count", [("kv_attend_kernel", 16), ("kv_weigh_kernel", 1), ("kv_append_kernel", 4),
                                        ("kv_evict_kernel", 6)])
def test_kernel_registers(kernels, name, count):  # noqa: F811
    mine = {k: v for k, v in kernels.items() if re.search(rf"\d+{name}[IE]", k)}
    assert len(mine) == count, sorted(mine)
    for k, v in mine.items():
        assert v["vgpr_spill_count"] == 0 and v["private_segment_fixed_size"] == 0 and v["agpr_count"] == 0, (k, v)
