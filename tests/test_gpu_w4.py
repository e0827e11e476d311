"""Packing of group-scaled 4-bit weights, dsq_linear_w4 and dsq_linear_w4a8 against the float64 oracle.

Tolerances, u = 2^-24, e = half a step of the output's type (relative).  A group's products are exact and added in
binary32 (at most 128 and the zero point's two operations), the groups' results added one after the other or in up
to 16 parts: with A the sum of |scale| (code + zero) |x|, at most (128 + 4 + G + 16) u A and e of the result, and
half the type's smallest step.  8-bit rows: a group's sum is an exact integer, (4 + G + 16) u A."""
import numpy as np
import pytest
import torch

from oracle import lm
from paper_1908_05033_amd import binding as B
from lm_helpers import DTYPES, U32, assert_within, code_rows, half_step, host, normal, pack, random_w4, tiny

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(1, 1), (16, 128), (17, 129), (5, 31), (130, 520), (256, 1024), (33, 4000)])
def test_pack(N, K, group):
    codes, scale, zero = random_w4(N + K, N, K, group)
    got = lm.unpack_w4(*[t.cpu().numpy() for t in pack(codes, scale, zero, group)], N, K, group)
    assert np.array_equal(got[0], codes) and np.array_equal(got[1], scale) and np.array_equal(got[2], zero)
    w = np.random.RandomState(K).randn(N, K).astype(np.float32) * 0.02
    w[0, :min(K, group)] = 0.0
    if N > 2:
        w[1] = np.abs(w[1])
        w[2] = -np.abs(w[2])
    want = lm.quantize_w4(w, group)
    got = lm.unpack_w4(*[t.cpu().numpy() for t in pack(None, None, None, group, w)], N, K, group)
    assert all(np.array_equal(a, b) for a, b in zip(got, want))
    # the recipe's rounding: at most half a step and the cut of the scale off
    step = np.repeat(got[1], group, 1)[:, :K]
    assert (np.abs(lm.levels(*got, group) - w) <= 0.5 * step * (1 + 1e-4) + 16 * step * 2.0 ** -20 + 0.5 * step).all()
    want = lm.quantize_w4(w, group, scale, zero)
    got = lm.unpack_w4(*[t.cpu().numpy() for t in pack(None, scale, zero, group, w)], N, K, group)
    assert all(np.array_equal(a, b) for a, b in zip(got, want))


def test_pack_saturates_and_keeps_20_bits():
    N, K, group = 16, 64, 32
    codes = np.full((N, K), 200, np.uint8)
    scale = np.random.RandomState(1).rand(N, 2).astype(np.float32)
    zero = np.full((N, 2), 99, np.uint8)
    c, s, z = lm.unpack_w4(*[t.cpu().numpy() for t in pack(codes, scale, zero, group)], N, K, group)
    assert (c == 15).all() and (z == 15).all()
    assert np.array_equal(s, lm.cut_scale(scale)) and (np.abs(s - scale) <= 2.0 ** -20 * scale).all()


def check(out, x, codes, scale, zero, group, bias=None, ints=False, rows=None):
    want, size = lm.linear(x, codes, scale, zero, group, None if bias is None else host(bias))
    G = scale.shape[1]
    bound = half_step(out.dtype) * np.abs(want) + tiny(out.dtype) + U32 * ((4 if ints else 132) + G + 16) * size
    got = host(out)
    assert_within(got, want, bound, "out")


def run_w4(x, packed, N, K, group, bias=None):
    out = torch.full((x.shape[0], N), 7.0, dtype=x.dtype, device="cuda")
    B.dsq_linear_w4(x, *packed, N, K, group, bias, out)
    torch.cuda.synchronize()
    return out


def run_w4a8(q, s, packed, N, K, group, dt, bias=None):
    out = torch.full((q.shape[0], N), 7.0, dtype=dt, device="cuda")
    B.dsq_linear_w4a8(q, s, *packed, N, K, group, bias, out)
    torch.cuda.synchronize()
    return out


MS = [1, 2, 15, 16, 17, 33, 64, 65, 100, 130, 257]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", MS)
def test_rows(M, dtype):
    for N, K, group in ((144, 1024, 128), (50, 520, 64)):
        c, s, z = random_w4(M, N, K, group)
        x, bias = normal(M, M, K, dtype=DTYPES[dtype]), normal(M + 1, N, dtype=DTYPES[dtype])
        check(run_w4(x, pack(c, s, z, group), N, K, group, bias), host(x), c, s, z, group, bias)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", MS)
def test_code_rows(M, dtype):
    for N, K, group in ((144, 1024, 128), (50, 520, 64)):
        c, s, z = random_w4(M, N, K, group)
        q, qs = code_rows(M, M, K)
        bias = normal(M + 1, N, dtype=DTYPES[dtype])
        check(run_w4a8(q, qs, pack(c, s, z, group), N, K, group, DTYPES[dtype], bias), host(q[:, :K]) * host(qs)[:, None], c, s, z,
              group, bias, ints=True)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(1, 1), (3, 8), (16, 127), (17, 128), (31, 129), (64, 33), (128, 2048), (129, 4097), (40, 9999), (1000, 300)])
def test_sizes(N, K, group):
    c, s, z = random_w4(N * K, N, K, group)
    p = pack(c, s, z, group)
    for M in (1, 5, 70, 200):
        for dt in DTYPES.values():
            x = normal(M, M, K, dtype=dt)
            check(run_w4(x, p, N, K, group), host(x), c, s, z, group)
        q, qs = code_rows(M, M, K, junk=True)            # (what lies behind K meets levels of 0)
        check(run_w4a8(q, qs, p, N, K, group, torch.float32), host(q[:, :K]) * host(qs)[:, None], c, s, z, group, ints=True)


def test_exact_sums():
    """Small integers: every sum is a binary32 integer, so the result is exact, zero points and all."""
    N, K, group = 48, 640, 64
    c, _, z = random_w4(3, N, K, group)
    s = np.full((N, K // group), 0.5, np.float32)
    p = pack(c, s, z, group)
    for M in (1, 20, 300):
        x = torch.from_numpy(np.random.RandomState(M).randint(-2, 3, (M, K)).astype(np.float32)).cuda()
        want = host(x) @ lm.levels(c, s, z, group).T
        assert np.array_equal(host(run_w4(x, p, N, K, group)), want)
        assert np.array_equal(host(run_w4(x.bfloat16(), p, N, K, group).float()), host(torch.from_numpy(want).bfloat16()))
        q = torch.zeros(M, B.dsq_code_row_bytes(K), dtype=torch.int8, device="cuda")
        q[:, :K] = x.to(torch.int8)
        assert np.array_equal(host(run_w4a8(q, torch.ones(M, device="cuda"), p, N, K, group, torch.float32)), want)


def test_every_code_and_every_zero_point():
    """One channel of x at a time: the level of each code under each zero point, in every type."""
    N, K, group = 256, 128, 128
    c = np.tile(np.arange(16, dtype=np.uint8), (N, K // 16))
    z = (np.arange(N) % 16).astype(np.uint8)[:, None]
    s = np.full((N, 1), 1.0, np.float32)
    p = pack(c, s, z, group)
    want = c.astype(np.float64) - z
    for dt in DTYPES.values():
        for lo in (0, 64):
            x = torch.zeros(64, K, dtype=dt, device="cuda")
            x[torch.arange(64), lo + torch.arange(64)] = 1.0
            assert np.array_equal(host(run_w4(x, p, N, K, group)), want[:, lo:lo + 64].T)


def test_extreme_codes():
    """-127 and 127 against levels of -15 and 15 over long rows: integer sums at their largest."""
    N, K, group = 32, 4096, 128
    c = np.zeros((N, K), np.uint8)
    c[::2] = 15
    z = np.zeros((N, K // group), np.uint8)
    z[1::2] = 15
    s = np.ones((N, K // group), np.float32)
    p = pack(c, s, z, group)
    for M in (3, 150):
        q = torch.full((M, K), 127, dtype=torch.int8, device="cuda")
        q[1::2] = -127
        want = host(q) @ lm.levels(c, s, z, group).T
        assert np.array_equal(host(run_w4a8(q, torch.ones(M, device="cuda"), p, N, K, group, torch.float32)), want)


@pytest.mark.parametrize("M", [1, 7, 150])
def test_strides_and_what_lies_between_rows(M):
    N, K, group = 70, 392, 32
    c, s, z = random_w4(1, N, K, group)
    p = pack(c, s, z, group)
    for dt in DTYPES.values():
        x = normal(1, M, K + 40, dtype=dt)[:, 16:16 + K]
        wide = torch.full((M + 1, N + 9), 5.0, dtype=dt, device="cuda")
        out = wide[:M, :N]
        B.dsq_linear_w4(x, *p, N, K, group, None, out)
        check(out.contiguous(), host(x), c, s, z, group)
        assert (wide[:, N:] == 5.0).all() and (wide[M] == 5.0).all()
        one = normal(2, 1, K, dtype=dt).expand(M, K)
        check(run_w4(one, p, N, K, group), host(one), c, s, z, group)
        q, qs = code_rows(3, M, K)
        wide.fill_(5.0)
        B.dsq_linear_w4a8(q, qs, *p, N, K, group, None, out)
        check(out.contiguous(), host(q[:, :K]) * host(qs)[:, None], c, s, z, group, ints=True)
        assert (wide[:, N:] == 5.0).all() and (wide[M] == 5.0).all()


@pytest.mark.parametrize("M", [4, 150])
def test_values_that_are_not_finite_stay_in_their_row(M):
    N, K, group = 48, 384, 64
    c, s, z = random_w4(1, N, K, group)
    p = pack(c, s, z, group)
    for dt in DTYPES.values():
        x = normal(1, M, K, dtype=dt)
        clean = run_w4(x, p, N, K, group)
        x[1, 7] = float("nan")
        x[2, 380] = float("inf")
        got = run_w4(x, p, N, K, group)
        assert torch.isnan(got[1]).all() and not torch.isfinite(got[2]).any()
        keep = [i for i in range(M) if i not in (1, 2)]
        assert torch.equal(got[keep], clean[keep])
        odd = torch.full((M,), 1.0, device="cuda")
        odd[1] = float("nan")                               # a row of dsq_rms_norm that was not finite
        q, _ = code_rows(2, M, K)
        q[1] = 0
        got = run_w4a8(q, odd, p, N, K, group, dt)
        assert torch.isnan(got[1]).all() and torch.isfinite(got[[i for i in range(M) if i != 1]]).all()


def test_small_and_large_activations():
    N, K, group = 33, 257, 32
    c, s, z = random_w4(1, N, K, group)
    p = pack(c, s, z, group)
    for M in (2, 150):
        for dt, scales in ((torch.float32, (1e-20, 1e-5, 1e25)), (torch.bfloat16, (1e-30, 1e30)), (torch.float16, (1e-6, 1e-4, 500.0))):
            for f in scales:
                x = normal(1, M, K).mul(f).to(dt)
                check(run_w4(x, p, N, K, group), host(x), c, s, z, group)


def test_no_rows():
    c, s, z = random_w4(1, 16, 64, 64)
    p = pack(c, s, z, 64)
    B.dsq_linear_w4(torch.empty(0, 64, device="cuda"), *p, 16, 64, 64, None, torch.empty(0, 16, device="cuda"))
    B.dsq_linear_w4a8(torch.empty(0, 128, dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda"), *p, 16, 64, 64, None,
                      torch.empty(0, 16, device="cuda"))
