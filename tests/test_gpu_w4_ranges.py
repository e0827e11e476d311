"""dsq_linear_w4 with activations near both ends of their type's range, in each kernel and tile.

Tolerances as derived in test_gpu_w4.py: they are relative to the sum A of |scale| (code + zero) |x| and to the result, and hold
wherever the result lies in the type's range, however large or small the sums of codes times x are on the way."""
import pytest
import torch

from lm_helpers import host, normal, pack, random_w4
from test_gpu_w4 import check, run_w4

pytestmark = pytest.mark.gpu

# rows and channels that take one row's kernel, the one of a few rows, and each tile
SHAPES = [(1, 40), (1, 9000), (5, 40), (16, 9230), (40, 48), (40, 4093), (256, 4093), (512, 4093), (900, 4093), (1024, 4224)]


def check_some(out, x, c, s, z, group, bias=None):
    """About 24 rows spread over all, the last among them."""
    at = sorted(set(range(0, x.shape[0], max(1, x.shape[0] // 24))) | {x.shape[0] - 1})
    check(out[at].contiguous(), host(x[at]), c, s, z, group, bias)


@pytest.mark.parametrize("M,N", SHAPES)
@pytest.mark.parametrize("K", [384, 640, 128])
def test_large_numbers_at_the_end_of_a_row(M, N, K):
    """Zeros but for the last eight channels: the sums of their codes and of theirs alone are below 2^128."""
    group = 128
    c, s, z = random_w4(1, N, K, group)
    p = pack(c, s, z, group)
    x = torch.zeros(M, K, device="cuda")
    x[:, -8:] = normal(3, M, 8).clamp(-2, 2) * 0.5e36 + 2e35
    assert 15 * 8 * float(x.abs().max()) < 2.0 ** 127
    for dt in (torch.bfloat16, torch.float32):
        check_some(run_w4(x.to(dt), p, N, K, group), x.to(dt), c, s, z, group)
