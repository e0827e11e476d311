"""dsq_linear_w4 with activations near both ends of their type's range, in each kernel and tile.

Tolerances as derived in test_gpu_w4.py: they are relative to the sum A of |scale| (code + zero) |x| and to the result, and hold
wherever the result lies in the type's range, however large or small the sums of codes times x are on the way."""
import numpy as np
import pytest
import torch

from lm_helpers import DTYPES, host, normal, pack, random_w4
from test_gpu_w4 import check, run_w4

pytestmark = pytest.mark.gpu

# rows and channels that take one row's kernel, the one of a few rows, and each tile
SHAPES = [(1, 40), (1, 9000), (5, 40), (16, 9230), (40, 48), (40, 4093), (256, 4093), (512, 4093), (900, 4093), (1024, 4224)]
# ... and the tiles of binary32 rows
SHAPES_F32 = [(1, 40), (1, 9000), (5, 40), (64, 4093), (2048, 640), (300, 12400)]


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


@pytest.mark.parametrize("M,N", SHAPES_F32)
@pytest.mark.parametrize("K,group", [(300, 64), (1024, 128), (100, 32), (7, 32)])
def test_binary32_numbers_below_the_parts_that_bfloat16_holds(M, N, K, group):
    c, s, z = random_w4(M, N, K, group)
    for up in (1.0, 2.0 ** 60):
        p = pack(c, s * np.float32(up), z, group)
        for f in (1e-33, 1e-35, 1e-37, 1e-38, 1e-40, 1e-43, 0.0):
            x = normal(M, M, K).double().mul(f).float()
            check_some(run_w4(x, p, N, K, group), x, c, s * np.float32(up), z, group)


@pytest.mark.parametrize("M,N", SHAPES_F32)
def test_small_and_ordinary_binary32_numbers_side_by_side(M, N):
    """A row of ordinary numbers beside rows of tiny ones, and tiny numbers in ordinary rows."""
    K, group = 520, 64
    c, s, z = random_w4(M, N, K, group)
    p = pack(c, s, z, group)
    x = normal(1, M, K).double()
    x[::2] *= 1e-37
    x[1::2, ::3] *= 1e-39
    x = x.float()
    check_some(run_w4(x, p, N, K, group), x, c, s, z, group)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K,group", [(300, 64), (1024, 128), (100, 32), (7, 32)])
def test_sums_of_codes_past_the_range(dtype, K, group):
    """Rows whose products with the codes pass 2^128 though the result does not."""
    dt = DTYPES[dtype]
    for M, N in SHAPES_F32 if dtype == "f32" else SHAPES:
        c, s, z = random_w4(M, N, K, group)
        s *= np.float32(2.0 ** -10)
        p = pack(c, s, z, group)
        for f in (1e28, 1e31, 1e34, 1e36, 5e37):
            x = normal(M, M, K).clamp(-5, 5).mul(f).to(dt)
            x[::3, :] = normal(M, M, K, dtype=dt)[::3]
            assert torch.isfinite(x).all()
            bias = normal(2, N, dtype=dt)
            check_some(run_w4(x, p, N, K, group, bias), x, c, s, z, group, bias)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_numbers_with_other_signs_and_a_result_past_the_range(dtype):
    """A result past the type's largest number is infinite, with its sign, and no other result is."""
    dt, K, group = DTYPES[dtype], 256, 64
    for M, N in SHAPES_F32 if dtype == "f32" else SHAPES:
        c, s, z = random_w4(M, N, K, group)
        c[:], z[:] = 15, 0
        s[:] = 2.0 ** -6
        s[1::2] = -2.0 ** -6
        s[2::4] = 2.0 ** -20
        p = pack(c, s, z, group)
        x = torch.full((M, K), 3e37, dtype=dt, device="cuda")
        out = run_w4(x, p, N, K, group)
        want = torch.full((N,), float("inf"), device="cuda")
        want[1::2] *= -1
        level = torch.arange(N, device="cuda") % 4 == 2
        assert torch.equal(out.float()[:, ~level], want[~level].expand(M, -1))
        assert torch.isfinite(out[:, level]).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_that_are_not_finite_beside_large_ones(dtype):
    dt, K, group = DTYPES[dtype], 300, 64
    big = 3e4 if dtype == "f16" else 1e37
    for M, N in SHAPES_F32 if dtype == "f32" else SHAPES:
        if M < 4:
            continue
        c, s, z = random_w4(M, N, K, group)
        s *= np.float32(2.0 ** -10)
        p = pack(c, s, z, group)
        x = normal(M, M, K).clamp(-2, 2).mul(big).to(dt)
        x[1, 5], x[2, 299], x[3] = float("nan"), float("inf"), float("-inf")
        out = run_w4(x, p, N, K, group)
        assert torch.isnan(out[1]).all() and not torch.isfinite(out[2]).any() and not torch.isfinite(out[3]).any()
        keep = [i for i in range(M) if i not in (1, 2, 3)]
        check_some(out[keep], x[keep], c, s, z, group)
