"""CPU: what the operators' kernel sources must not hold."""
import os
import re

import pytest

from paper_2606_05613_gb300 import build as nb

# kernels that may begin before the one that writes their inputs has ended (launch_behind)
BEHIND = ["gate.cu", "gate_few.cu", "adamw.cu", "tile_gemm.cuh", "tensor_core.cuh", "tile_host.cu"]


@pytest.mark.parametrize("name", BEHIND)
def test_kernels_launched_behind_others_do_not_read_by_the_read_only_path(name):
    """ld.global.nc, and __ldg with it, is for memory that nothing writes while the kernel
    runs; its order against the wait for the kernel ahead is not defined."""
    with open(os.path.join(nb.CSRC, name)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    assert "__ldg" not in code and not re.search(r"ld\.global(\.[a-z0-9:_]+)*\.nc", code) and "ld16_nc" not in code
