"""Each kernel and tile that dsq_linear_w4 and dsq_linear_w4a8 choose from, at the edges of its rows, channels and blocks of
input channels, and offsets past 32 bits.

Tolerances as derived in test_gpu_w4.py; a row alone and a few rows add up to 16 parts, tiles up to 4: within its 16."""
import numpy as np
import pytest
import torch

from oracle import lm
from paper_1908_05033_amd import binding as B
from lm_helpers import DTYPES, code_rows, host, normal, pack, random_w4
from test_gpu_w4 import check, run_w4, run_w4a8

pytestmark = pytest.mark.gpu


def both(M, N, K, group, dtypes=DTYPES):
    c, s, z = random_w4(M + N + K, N, K, group)
    p = pack(c, s, z, group)
    for name in dtypes:
        dt = DTYPES[name]
        x, bias = normal(M, M, K, dtype=dt), normal(N, N, dtype=dt)
        check(run_w4(x, p, N, K, group, bias), host(x), c, s, z, group, bias)
    q, qs = code_rows(M, M, K, junk=True)
    check(run_w4a8(q, qs, p, N, K, group, torch.bfloat16), host(q[:, :K]) * host(qs)[:, None], c, s, z, group, ints=True)


# (rows and channels of each tile, one row and three channels short of whole ones; channels 1100: an odd number of
# iterations in every tile and an end inside a block; 264: fewer blocks than waves share; 100: less than one)
@pytest.mark.parametrize("K", [100, 264, 1100])
@pytest.mark.parametrize("M,N", [(31, 4093), (127, 4093), (255, 4093), (511, 4093), (1023, 4093)])
def test_tiles(M, N, K):
    both(M, N, K, {100: 32, 264: 64, 1100: 128}[K])


@pytest.mark.parametrize("K,group", [(264, 32), (390, 64), (128, 128)])
def test_the_largest_tile(K, group):
    both(2047, 8189, K, group, ("bf16", "f16"))


@pytest.mark.parametrize("group", [32, 64, 128])
def test_every_tile_in_every_group_size(group):
    for M, N in ((40, 4096), (256, 4096), (512, 4096), (1024, 4096)):
        both(M, N, 387, group)


# one, two and four tiles of output channels a wave
@pytest.mark.parametrize("N", [50, 4603, 4620, 9210, 9230])
@pytest.mark.parametrize("M", [2, 3, 16])
def test_a_few_rows(M, N):
    both(M, N, 136, 32)
    both(M, N, 1290, 128)


# one to eight waves a tile of output channels; rows of one segment and of several
@pytest.mark.parametrize("N,K", [(20, 8200), (20, 70000), (5000, 2100), (9000, 2100), (17000, 1300), (33000, 1300), (66000, 4100)])
def test_one_row(N, K):
    both(1, N, K, 128 if N > 10000 else 32)


@pytest.mark.parametrize("K", [1, 7, 8, 9, 15])
@pytest.mark.parametrize("M", [1, 3, 40, 300])
def test_fewer_input_channels_than_a_load(M, K):
    both(M, 37, K, 32)


def test_more_rows_than_a_launch_holds():
    """Rows of five channels take the kernel for a few rows, 2^19 of them a launch."""
    M, N, K, group = (1 << 20) + 77, 19, 5, 64
    c, s, z = random_w4(1, N, K, group)
    p = pack(c, s, z, group)
    at = torch.tensor([0, 1, 15, 16, (1 << 19) - 1, 1 << 19, (1 << 20) - 1, 1 << 20, M - 1], device="cuda")
    for dt in (torch.bfloat16, torch.float32):
        x = torch.randn(M, K, device="cuda").to(dt)
        out = run_w4(x, p, N, K, group)
        check(out[at], host(x[at]), c, s, z, group)
        assert not (out == 7.0).all(1).any()


def test_subnormal_activations():
    """The smallest numbers of a type count in the products and in the sums for the zero points."""
    N, K, group = 40, 300, 64
    c, _, z = random_w4(2, N, K, group)
    for dt, scale in ((torch.float16, 2.0 ** 10), (torch.bfloat16, 2.0 ** 100)):
        s = np.full((N, -(-K // group)), scale, np.float32)
        p = pack(c, s, z, group)
        for M in (1, 5, 100):
            rs = np.random.RandomState(M)
            x = torch.from_numpy(rs.randint(-100, 101, (M, K)).astype(np.float64) * torch.finfo(dt).smallest_normal * torch.finfo(dt).eps).to(dt).cuda()
            assert (x != 0).float().mean() > 0.9
            check(run_w4(x, p, N, K, group), host(x), c, s, z, group)


def test_scales_of_zero_and_negative_ones():
    N, K, group = 37, 260, 64
    c, s, z = random_w4(4, N, K, group)
    s[::3] = 0.0
    s[1::3] *= -1.0
    p = pack(c, s, z, group)
    for M in (1, 6, 90):
        for dt in DTYPES.values():
            x = normal(M, M, K, dtype=dt)
            out = run_w4(x, p, N, K, group)
            check(out, host(x), c, s, z, group)
            assert not out[:, ::3].any()
        q, qs = code_rows(M, M, K)
        check(run_w4a8(q, qs, p, N, K, group, torch.float32), host(q[:, :K]) * host(qs)[:, None], c, s, z, group, ints=True)


def test_more_than_2_32_bytes_of_weights():
    """The last channels of a layer whose codes take 4.4 GB."""
    N, K, group, tail = (1 << 20) + 128, 8320, 128, 128
    c, s, z = random_w4(5, tail, K, group)
    few = pack(c, s, z, group)
    w = torch.zeros(B.dsq_w4_packed_bytes(N, K), dtype=torch.uint8, device="cuda")
    sc = torch.zeros(B.dsq_w4_scale_bytes(N, K, group), dtype=torch.uint8, device="cuda")
    w[-few[0].numel():] = few[0]
    sc[-few[1].numel():] = few[1]
    for M in (1, 4, 40):
        for dt in (torch.bfloat16, torch.float32):
            x = normal(M, M, K, dtype=dt)
            out = run_w4(x, (w, sc), N, K, group)
            check(out[:, -tail:].contiguous(), host(x), c, s, z, group)
            assert not out[:, :-tail].any()
        q, qs = code_rows(M, M, K)
        out = run_w4a8(q, qs, (w, sc), N, K, group, torch.bfloat16)
        check(out[:, -tail:].contiguous(), host(q[:, :K]) * host(qs)[:, None], c, s, z, group, ints=True)
        assert not out[:, :-tail].any()


@pytest.mark.parametrize("M", [5, 40])
def test_rows_more_than_2_32_bytes_apart(M):
    N, K, group, far = 50, 200, 64, 125_000_003
    c, s, z = random_w4(6, N, K, group)
    p = pack(c, s, z, group)
    if M == 5:
        far *= 8
    big = torch.empty((M - 1) * far + 512, dtype=torch.bfloat16, device="cuda")
    x, out = big.as_strided((M, K), (far, 1)), big.as_strided((M, N), (far, 1), 256)
    x.copy_(normal(M, M, K, dtype=torch.bfloat16))
    B.dsq_linear_w4(x, *p, N, K, group, None, out)
    check(out.contiguous(), host(x), c, s, z, group)


def test_outputs_of_codes_more_than_2_32_bytes_apart():
    M, N, K, group, far = 40, 50, 200, 64, 125_000_003
    c, s, z = random_w4(7, N, K, group)
    p = pack(c, s, z, group)
    q, qs = code_rows(1, M, K)
    big = torch.empty((M - 1) * far + 64, dtype=torch.float16, device="cuda")
    out = big.as_strided((M, N), (far, 1))
    B.dsq_linear_w4a8(q, qs, *p, N, K, group, None, out)
    check(out.contiguous(), host(q[:, :K]) * host(qs)[:, None], c, s, z, group, ints=True)


@pytest.mark.parametrize("M", [3, 40, 300])
def test_results_do_not_depend_on_what_lies_behind_the_rows(M):
    """Memory behind the last row and behind each row's end, full of NaN."""
    N, K, group = 70, 260, 64
    c, s, z = random_w4(8, N, K, group)
    p = pack(c, s, z, group)
    for dt in DTYPES.values():
        wide = torch.full((M + 40, K + 29), float("nan"), dtype=dt, device="cuda")
        x = wide[:M, :K]
        x.copy_(normal(1, M, K, dtype=dt))
        check(run_w4(x, p, N, K, group), host(x), c, s, z, group)
