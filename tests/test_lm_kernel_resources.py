"""Register budget of the compiled language-model kernels (host-side check, no GPU): the products do not spill at all; of the
norm, rows of more than eight elements a thread (over 8192 16-bit or 4096 binary32 ones) leave some in scratch memory."""
import os
import re

import pytest

from test_kernel_resources import CSRC, _device_asm


@pytest.mark.parametrize("source", ["rms_norm.hip", "w4_pack.hip", "w4_row.hip", "w4_rows.hip", "w4_tiles.hip"])
def test_kernels_stay_inside_their_registers(source):
    asm = _device_asm(os.path.join(CSRC, source))
    kernels = re.findall(r"\.name:\s+(\S+).*?\.private_segment_fixed_size:\s+(\d+).*?\.vgpr_spill_count:\s+(\d+)", asm, re.S)
    assert kernels, "no kernel metadata found in the device assembly"
    allowed = 64 if source == "rms_norm.hip" else 0
    assert not [k for k in kernels if int(k[2]) > allowed or int(k[1]) > 4 * allowed]
    few = [k for k in kernels if "ELi1024ELi2E" not in k[0] and "ELi1024ELi4E" not in k[0]]
    assert not [k for k in few if int(k[1]) or int(k[2])]
    # (the packed additions, products and fused ones of binary32 are not to be used)
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", asm)
