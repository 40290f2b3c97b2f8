"""Which instances of the microscaled kernels spill registers (read from the built library; no GPU needed): those that are known to, and no others."""
import re

import pytest

from paper_2312_08656_amd import binding
from test_scratch import code_objects

# numbers of an instance's template arguments as they stand in its name, and how many there are of them
KNOWN = {
    "quantize_kernel": [], "dequantize_kernel": [], "linear_long_kernel": [], "add_ranges_kernel": [],
    "linear_kernel": [r"^8 0 1 [01]$"],  # 513 to 1024 columns in, fp32 Y in 16-byte pieces
    "weight_grad_kernel": [r"^8 1 1 2 [01] 1 8$"],  # 64 x 64, two-byte columns, k above 32
    "input_grad_kernel": [r"^32 1 8 1 ([12] [48]|[4357] 1) 0$",  # dH of 385 to 512 columns: every form but bf16 and fp16 in 16-byte pieces
                          r"^16 2 4 2 ([01] 8|[357] 1) 0$",      # 129 to 256 at din above 128: k above 32, rows that come element by element
                          r"^24 1 4 2 [357] 1 0$"],              # 257 to 384: rows that come element by element
}


@pytest.fixture(scope="module")
def kernels():
    if not binding.lib_path().exists():
        from paper_2312_08656_amd import build
        build.build()
    found = []
    for name, scratch, spilled in code_objects(binding.lib_path().read_bytes()):
        m = re.search(r"\d([a-z_]+_kernel)I(.*?)EEv", name)
        if m and m.group(1) in KNOWN:
            found.append((m.group(1), " ".join(re.findall(r"(?:Li|Lb|LNS0_4RowsE)(\d+)", m.group(2))), scratch, spilled))
    return found


@pytest.mark.parametrize("kernel,least", [("quantize_kernel", 18), ("dequantize_kernel", 18), ("linear_kernel", 30), ("linear_long_kernel", 3), ("weight_grad_kernel", 70),
                                          ("add_ranges_kernel", 3), ("input_grad_kernel", 90)])
def test_no_other_instance_spills(kernels, kernel, least):
    mine = [k for k in kernels if k[0] == kernel]
    assert len(mine) >= least
    spilling = [k for k in mine if k[2] or k[3]]
    assert [k for k in spilling if not any(re.match(known, k[1]) for known in KNOWN[kernel])] == []
    assert all(k[3] <= 52 for k in spilling)
