"""What the RMS norm's kernels leave in scratch memory, kernel by kernel (host-side check, no GPU): nothing with one vector a thread;
with several the forward pass a few registers, the backward pass of 16-bit rows none and that of binary32 rows of more than 8192
numbers, at four vectors a thread, about fifty."""
import os
import re

from test_kernel_resources import CSRC, _device_asm


def allowed(kernel):
    backward, vectors = "bwd" in kernel, re.search(r"kernelILi(\d)ELi(\d+)ELi(\d)E", kernel)
    if not vectors or vectors.group(3) == "1":
        return 0
    if not backward:
        return 8
    return 56 if vectors.group(1) == "0" and vectors.group(3) == "4" else 0


def test_spilled_registers_of_each_kernel():
    asm = _device_asm(os.path.join(CSRC, "rms_norm.hip"))
    kernels = re.findall(r"\.name:\s+(\S+).*?\.vgpr_count:\s+(\d+).*?\.vgpr_spill_count:\s+(\d+)", asm, re.S)
    assert len([k for k in kernels if "kernelILi0ELi1024ELi4E" in k[0]]) == 4          # (forward and backward, whole and odd rows)
    over = [(name, int(spilled)) for name, _, spilled in kernels if int(spilled) > allowed(name)]
    assert not over, over
    # workgroups of 1024 threads need 128 registers a lane or fewer
    assert not [k for k in kernels if "ELi1024E" in k[0] and int(k[1]) > 128]
