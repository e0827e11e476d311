"""Register budget of the compiled kernels for heads (host-side check, no GPU): nothing in scratch memory but one or two registers outside
the loops of three kernels that use all of theirs, and as many waves a SIMD as the kernels' comments say."""
import os
import re

import pytest

from test_kernel_resources import CSRC, _device_asm

FULL = ("attn_fwd_kernelIDF16_Li128ELi4E", "attn_fwd_kernelIDF16bLi128ELi4E", "attn_bwd_q_kernelIDF16_Li128ELi4E", "attn_bwd_q_kernelIDF16bLi128ELi4E",
        "attn_bwd_q_kernelIfLi128ELi1E")


@pytest.mark.parametrize("source,count", [("head_rope.hip", 31), ("attn_fwd.hip", 18), ("attn_bwd.hip", 30), ("attn_cache.hip", 33)])
def test_kernels_stay_inside_their_registers(source, count):
    asm = _device_asm(os.path.join(CSRC, source))
    kernels = re.findall(r"\.name:\s+(\S+).*?\.private_segment_fixed_size:\s+(\d+).*?\.vgpr_count:\s+(\d+).*?\.vgpr_spill_count:\s+(\d+)", asm, re.S)
    assert len(kernels) == count
    for name, scratch, _, spilled in kernels:
        full = any(f in name for f in FULL)
        assert int(spilled) <= (2 if full else 0) and int(scratch) <= (16 if full else 0), (name, scratch, spilled)
    # (the packed additions, products and fused ones of binary32 are not to be used)
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", asm)
    # nothing is spilled between the first and the last product of a kernel
    for fn in re.split(r"\n(?=_Z\S+:)", asm):
        lines = [l.split()[0] for l in fn.splitlines() if l.startswith("\t") and not l.startswith("\t.") and l.split()]
        products = [i for i, l in enumerate(lines) if l.startswith("v_mfma")]
        if products:
            assert not any(l.startswith("scratch_") for l in lines[products[0]:products[-1]]), fn.split(":", 1)[0]


@pytest.mark.parametrize("source,kernel,most", [("attn_fwd.hip", r"attn_fwd_kernelIDF16b?_?Li\d+ELi4E", 256), ("attn_bwd.hip", r"attn_bwd_q_kernelIDF16b?_?Li\d+ELi4E", 256),
                                                ("attn_bwd.hip", r"attn_bwd_k_kernelIDF16b?_?", 256), ("attn_cache.hip", r"attn_cache_(tiles_)?kernelIDF16b?_?", 256),
                                                ("head_rope.hip", r"head_rope_kernelI", 64), ("head_rope.hip", r"head_rope_bwd_kernelI", 168)])
def test_waves_a_simd(source, kernel, most):
    """Two waves of 256 registers, eight of 64, three of 168."""
    asm = _device_asm(os.path.join(CSRC, source))
    kernels = re.findall(r"\.name:\s+(\S+).*?\.vgpr_count:\s+(\d+)", asm, re.S)
    mine = [(n, int(v)) for n, v in kernels if re.search(kernel, n)]
    assert len(mine) >= 4 and all(v <= most for _, v in mine), mine
