"""Registers of the prompt kernels for heads of up to 64 elements (host-side check, no GPU): what follows their loops, rows that are not finite among it, does
not cost the loops a wave a SIMD."""
import os
import re

import pytest

from test_kernel_resources import CSRC, _device_asm


@pytest.mark.parametrize("kernel,most", [(r"attn_fwd_kernelIDF16b?_?Li64ELi4E", 128), (r"attn_fwd_kernelIfLi64ELi4E", 168)])
def test_waves(kernel, most):
    """Four waves of 128 registers, three of 168."""
    kernels = re.findall(r"\.name:\s+(\S+).*?\.vgpr_count:\s+(\d+)", _device_asm(os.path.join(CSRC, "attn_fwd.hip")), re.S)
    mine = [(n, int(v)) for n, v in kernels if re.search(kernel, n)]
    assert mine and all(v <= most for _, v in mine), mine
