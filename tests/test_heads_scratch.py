"""Which instances of the norm's, the class rows' and the few-row product's kernels spill registers (read from the built library; no GPU needed): one."""
import re

import pytest

from paper_2312_08656_amd import binding
from test_scratch import code_objects

LEAST = {"norm_kernel": 39, "norm_grad_kernel": 39, "add_parts_kernel": 1, "class_team_kernel": 100, "class_lane_kernel": 12, "class_own_kernel": 18, "class_held_kernel": 75, "class_rows_kernel": 45, "class_parts_kernel": 9,
         "class_join_kernel": 6, "class_gradient_kernel": 6, "matvec_kernel": 6, "matvec_lanes_kernel": 40}

KNOWN = "norm_grad_kernelILi0ELi1024ELi2E"  # fp32 rows of 8193 to 16384 columns: 2 registers


@pytest.fixture(scope="module")
def kernels():
    if not binding.lib_path().exists():
        from paper_2312_08656_amd import build
        build.build()
    found = {}
    for name, scratch, spilled in code_objects(binding.lib_path().read_bytes()):
        m = re.search(r"\d([a-z_]+_kernel)(I|E)", name)
        if m and m.group(1) in LEAST:
            found.setdefault(m.group(1), []).append((name, scratch, spilled))
    return found


@pytest.mark.parametrize("kernel", LEAST)
def test_no_other_instance_spills(kernels, kernel):
    assert len(kernels[kernel]) >= LEAST[kernel]
    assert [k for k in kernels[kernel] if (k[1] or k[2]) and not (KNOWN in k[0] and k[2] <= 2)] == []
