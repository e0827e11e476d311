"""dsq_linear_w4 and dsq_linear_w4a8 where workgroups of 256 output channels meet packed weights that end after 128 of them.
Tolerances as derived in test_gpu_w4.py."""
import pytest
import torch

from paper_1908_05033_amd import binding as B
from lm_helpers import DTYPES, code_rows, host, normal, pack, random_w4
from test_gpu_w4 import check, run_w4, run_w4a8

pytestmark = pytest.mark.gpu

# type (0: 16-bit rows, 1: 8-bit rows, 2: binary32 ones), rows, channels, rows of the tile that such a call takes
CASES = [(0, 512, 5504, 64), (0, 511, 5377, 64), (0, 1024, 4224, 128), (0, 129, 29568, 128), (1, 512, 5500, 64), (1, 1024, 4224, 128),
         (1, 257, 29500, 64), (2, 2048, 640, 32), (2, 300, 12400, 64)]


@pytest.mark.parametrize("kind,M,N", [c[:3] for c in CASES])
def test_channels_end_inside_a_workgroup(kind, M, N):
    for K, group in ((128, 128), (330, 32)):
        c, s, z = random_w4(M + N, N, K, group)
        p = pack(c, s, z, group)
        if kind == 1:
            q, qs = code_rows(M, M, K)
            check(run_w4a8(q, qs, p, N, K, group, torch.bfloat16), host(q[:, :K]) * host(qs)[:, None], c, s, z, group, ints=True)
            continue
        for dt in (DTYPES["f32"],) if kind == 2 else (DTYPES["bf16"], DTYPES["f16"]):
            x, bias = normal(M, M, K, dtype=dt), normal(N, N, dtype=dt)
            check(run_w4(x, p, N, K, group, bias), host(x), c, s, z, group, bias)
