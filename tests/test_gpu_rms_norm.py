"""dsq_rms_norm and dsq_rms_norm_bwd against the float64 oracle.

Tolerances, u = 2^-24, e = half a step of the type (relative):
  sum      the binary32 sum rounded to the type: equal bit for bit
  y        formed in binary64, rounded to binary32 and to the type: e + u of the value, half the smallest step below it
  codes    the definition is exact: equal
  scale, rstd   one rounding from binary64 and a few of 2^-53: 2u of the value
  grad_x   binary32, with m = mean of (t * n): each of r*t, r*n*m has at most four roundings, m at most 64 + log2(threads)
           + 3 of its terms' absolute mean (a thread adds at most 32 products, or dim / 1024 in rows longer than the
           registers), and the result's own
  grad_weight   a workgroup adds the rows it takes one after the other in binary32, the rest is binary64: rows taken + 16
           roundings of the absolute sum"""
import numpy as np
import pytest
import torch

from oracle import lm
from paper_1908_05033_amd import binding as B
from lm_helpers import DTYPES, U32, assert_within, half_step, host, normal, tiny

pytestmark = pytest.mark.gpu
EPS = 1e-5

# every number of threads a row, vectors a thread, and the kernel for longer rows; odd lengths end inside a vector
DIMS = [1, 2, 7, 8, 64, 127, 128, 200, 251, 512, 513, 1000, 1024, 1031, 2048, 2050, 4096, 4099, 8192, 8200, 16384, 16391,
        32768, 32771, 40000]


def run_fwd(x, res, w, want=("sum", "y", "codes", "scales", "rstd"), eps=EPS):
    rows, dim = x.shape
    out = {"sum": torch.empty(rows, dim, dtype=x.dtype, device="cuda"), "y": torch.empty(rows, dim, dtype=x.dtype, device="cuda"),
           "codes": torch.full((rows, B.dsq_code_row_bytes(dim)), 99, dtype=torch.int8, device="cuda"),
           "scales": torch.full((rows,), 7.0, device="cuda"), "rstd": torch.full((rows,), 7.0, device="cuda")}
    out = {k: v if k in want else None for k, v in out.items()}
    B.dsq_rms_norm(x, res, w, eps, out["sum"], out["y"], out["codes"], out["scales"], out["rstd"])
    torch.cuda.synchronize()
    return out


def check_fwd(x, res, w, out, eps=EPS):
    dt, dim = x.dtype, x.shape[1]
    h = (x.float() + res.float()).to(dt) if res is not None else x
    hd, wd = host(h), host(w) if w is not None else np.ones(dim)
    y, r = lm.rms_norm(hd, wd, eps)
    if out["sum"] is not None:
        assert torch.equal(out["sum"], h)
    if out["y"] is not None:
        assert_within(host(out["y"]), y, (half_step(dt) + 2 * U32) * np.abs(y) + tiny(dt), "y")
    if out["rstd"] is not None:
        assert_within(host(out["rstd"]), r, 2 * U32 * r, "rstd")
    if out["codes"] is not None:
        codes, scale = lm.code_rows(hd, wd, r)
        got = out["codes"].cpu().numpy()
        assert np.array_equal(got[:, :dim], codes)
        assert not got[:, dim:].any()
        assert_within(host(out["scales"]), scale, 2 * U32 * scale, "scale")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", DIMS)
def test_forward(dim, dtype):
    dt = DTYPES[dtype]
    rows = 37 if dim <= 4096 else 3
    x, res, w = normal(dim, rows, dim, dtype=dt), normal(dim + 1, rows, dim, dtype=dt, scale=3.0), normal(dim + 2, dim, dtype=dt)
    check_fwd(x, res, w, run_fwd(x, res, w))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 1000])
def test_rows(rows, dtype):
    dt = DTYPES[dtype]
    for dim in (96, 1536):
        x, w = normal(rows, rows, dim, dtype=dt), normal(rows + 2, dim, dtype=dt)
        check_fwd(x, None, w, run_fwd(x, None, w))


@pytest.mark.parametrize("want", [("sum",), ("y",), ("codes", "scales"), ("rstd",), ("sum", "codes", "scales"), ("y", "rstd")])
@pytest.mark.parametrize("dim", [320, 33000])
def test_each_output_alone(dim, want):
    x, res = normal(3, 5, dim, dtype=torch.bfloat16), normal(4, 5, dim, dtype=torch.bfloat16)
    for r in (res, None):
        for w in (normal(5, dim, dtype=torch.bfloat16), None):
            check_fwd(x, r, w, run_fwd(x, r, w, want))


@pytest.mark.parametrize("dim", [264, 4096, 33000])
def test_rows_that_lie_apart_and_a_row_that_repeats(dim):
    for dt in DTYPES.values():
        wide, w = normal(1, 6, dim + 24, dtype=dt), normal(2, dim, dtype=dt)
        x, res = wide[:, 8:8 + dim], normal(3, 1, dim, dtype=dt).expand(6, dim)
        check_fwd(x, res, w, run_fwd(x, res, w))


@pytest.mark.parametrize("dim", [72, 4099, 33000])
@pytest.mark.parametrize("place", ["x", "residual"])
def test_sum_in_the_place_of_an_input(place, dim):
    dt = torch.bfloat16
    x, res, w = normal(1, 9, dim, dtype=dt), normal(2, 9, dim, dtype=dt), normal(3, dim, dtype=dt)
    want = run_fwd(x, res, w)
    y, s = torch.empty_like(x), x if place == "x" else res
    B.dsq_rms_norm(x, res, w, EPS, s, y, None, None, None)
    assert torch.equal(s, want["sum"]) and torch.equal(y, want["y"])
    x = normal(1, 9, dim, dtype=dt)
    res = normal(2, 9, dim, dtype=dt)
    B.dsq_rms_norm(x, res, w, EPS, res, x, None, None, None)         # both in place
    assert torch.equal(res, want["sum"]) and torch.equal(x, want["y"])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [128, 3000, 33000])
def test_codes_at_halves(dim, dtype):
    """Quotients on a half and one step of the type beside it: the code is the exact quotient's."""
    dt = DTYPES[dtype]
    rs = np.random.RandomState(5)
    top = 127.0 * 4
    h = (rs.randint(-126, 127, (7, dim)) + 0.5) * 4.0                # 127 h / amax is a half exactly
    h[:, 0] = top
    h = torch.from_numpy(h).to(dt)
    near = h.clone()
    bits = near[:, 1::2].contiguous().view(torch.int32 if dt == torch.float32 else torch.int16) + torch.from_numpy(
        rs.choice([-1, 1], near[:, 1::2].shape)).to(torch.int32 if dt == torch.float32 else torch.int16)
    near[:, 1::2] = bits.view(dt)
    near = torch.where(near.abs() > top, h, near)
    for x in (h.cuda(), near.cuda()):
        w = torch.ones(dim, dtype=dt, device="cuda")
        check_fwd(x, None, w, run_fwd(x, None, w))


@pytest.mark.parametrize("dim", [100, 5000, 33000])
def test_magnitudes(dim):
    """Rows of tiny and huge numbers: squares and products stay inside binary64."""
    for dt, scales in ((torch.float32, (1e-38, 1e-30, 1e-6, 1e18, 1e37)), (torch.bfloat16, (1e-36, 1e20, 1e37)), (torch.float16, (1e-5, 1e4))):
        x = torch.cat([normal(i, 1, dim).clamp(-3, 3).mul(s).to(dt) for i, s in enumerate(scales)])
        w = normal(9, dim, dtype=dt)
        out = run_fwd(x, None, w, eps=1e-30)
        # (1/rms of the largest rows is below binary32's normal numbers, as is the smallest rows' scale: absolute steps of 2^-150)
        r = lm.rms_norm(host(x), host(w), 1e-30)[1]
        assert_within(host(out["rstd"]), r, 2 * U32 * r + 2.0 ** -149, "rstd")
        y = lm.rms_norm(host(x), host(w), 1e-30)[0]
        assert_within(host(out["y"]), y, (half_step(dt) + 2 * U32) * np.abs(y) + tiny(dt) + 2.0 ** -149, "y")
        assert np.array_equal(out["codes"].cpu().numpy()[:, :dim], lm.code_rows(host(x), host(w), r)[0])


@pytest.mark.parametrize("dim", [24, 300, 5000, 33000])
def test_rows_of_zeros_and_rows_that_are_not_finite(dim):
    for dt in DTYPES.values():
        x, w = normal(1, 8, dim, dtype=dt), normal(2, dim, dtype=dt)
        clean = run_fwd(x, None, w)
        x[1] = 0
        x[3, dim // 2] = float("inf")
        x[5, dim - 1] = float("nan")
        x[6, 0] = -float("inf")
        out = run_fwd(x, None, w)
        assert not out["y"][1].any() and not out["codes"][1].any() and out["scales"][1] == 0
        for row in (3, 5, 6):
            assert torch.isnan(out["scales"][row]) and not out["codes"][row].any()
            assert torch.isnan(out["y"][row]).any()
        for row in (0, 2, 4, 7):
            assert all(torch.equal(out[k][row], clean[k][row]) for k in out)
        for odd in (float("nan"), float("inf")):
            w2 = w.clone()
            w2[dim // 3] = odd
            x2 = normal(1, 8, dim, dtype=dt)
            x2[2, dim // 3] = 0
            out = run_fwd(x2, None, w2)
            assert torch.isnan(out["scales"]).all() and not out["codes"].any()


def run_bwd(h, w, rstd, gy, gs, with_gw=True):
    rows, dim = h.shape
    gx = torch.empty(rows, dim, dtype=h.dtype, device="cuda")
    gw = torch.full((dim,), 7.0, device="cuda") if with_gw else None
    ws = torch.full((B.dsq_rms_norm_bwd_bytes(rows, dim),), 0x7F, dtype=torch.uint8, device="cuda") if with_gw else None
    B.dsq_rms_norm_bwd(h, w, rstd, gy, gs, gx, gw, ws)
    torch.cuda.synchronize()
    return gx, gw


def check_bwd(h, w, rstd, gy, gs, gx, gw):
    dt, (rows, dim) = h.dtype, h.shape
    hd, wd, r, gyd = host(h), host(w) if w is not None else np.ones(dim), host(rstd), host(gy)
    gsd = host(gs) if gs is not None else None
    want_x, want_w = lm.rms_norm_grads(hd, wd, r, gyd, gsd)
    n, t = hd * r[:, None], gyd * wd
    m = np.abs((t * n).mean(axis=1, keepdims=True))
    size = r[:, None] * (np.abs(t) + np.abs(n) * m) + (np.abs(gsd) if gs is not None else 0)
    adds = 64 + 10 + 3 + dim // 1024
    bound = half_step(dt) * np.abs(want_x) + tiny(dt) + U32 * (6 * size + adds * (r[:, None] * np.abs(n)) * np.abs(t * n).mean(axis=1, keepdims=True))
    assert_within(host(gx), want_x, bound, "grad_x")
    if gw is not None:
        taken = -(-rows // 512) + 16
        assert_within(host(gw), want_w, U32 * (taken + 3) * np.abs(gyd * n).sum(axis=0), "grad_weight")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", DIMS)
def test_backward(dim, dtype):
    dt = DTYPES[dtype]
    rows = 41 if dim <= 4096 else 3
    h, w = normal(dim, rows, dim, dtype=dt, scale=2.0), normal(dim + 2, dim, dtype=dt)
    gy, gs = normal(dim + 3, rows, dim, dtype=dt), normal(dim + 4, rows, dim, dtype=dt)
    rstd = run_fwd(h, None, w, ("rstd",))["rstd"]
    check_bwd(h, w, rstd, gy, gs, *run_bwd(h, w, rstd, gy, gs))
    check_bwd(h, None, rstd, gy, None, *run_bwd(h, None, rstd, gy, None, dim % 2 == 0))


@pytest.mark.parametrize("rows", [1, 511, 512, 513, 9000])
def test_backward_of_many_rows(rows):
    """More rows than workgroups: each takes several, and the result is the same every time."""
    for dim, dt in ((64, torch.float32), (1000, torch.bfloat16), (5000, torch.float16)):
        h, w = normal(1, rows, dim, dtype=dt), normal(2, dim, dtype=dt)
        gy, gs = normal(3, rows, dim, dtype=dt), normal(4, rows, dim, dtype=dt)
        rstd = run_fwd(h, None, w, ("rstd",))["rstd"]
        gx, gw = run_bwd(h, w, rstd, gy, gs)
        check_bwd(h, w, rstd, gy, gs, gx, gw)
        again = run_bwd(h, w, rstd, gy, gs)
        assert torch.equal(gx, again[0]) and torch.equal(gw, again[1])


def test_backward_of_long_rows_takes_several_rows_a_workgroup():
    rows, dim = 1030, 16400                                   # float32 rows past the registers of a workgroup
    h, w = normal(1, rows, dim), normal(2, dim)
    gy = normal(3, rows, dim)
    rstd = run_fwd(h, None, w, ("rstd",))["rstd"]
    check_bwd(h, w, rstd, gy, None, *run_bwd(h, w, rstd, gy, None))


def test_backward_against_differences():
    """The kernel's gradients against central differences of the float64 oracle, along random directions."""
    rows, dim, step = 6, 515, 1e-6
    h, w = normal(1, rows, dim), normal(2, dim)
    gy, gs = normal(3, rows, dim), normal(4, rows, dim)
    rstd = run_fwd(h, None, w, ("rstd",))["rstd"]
    gx, gw = run_bwd(h, w, rstd, gy, gs)
    hd, wd, gyd, gsd = host(h), host(w), host(gy), host(gs)
    loss = lambda a, b: (gyd * lm.rms_norm(a, b, EPS)[0]).sum() + (gsd * a).sum()
    rs = np.random.RandomState(1)
    for _ in range(5):
        d = rs.randn(rows, dim)
        diff = (loss(hd + step * d, wd) - loss(hd - step * d, wd)) / (2 * step)
        assert abs(diff - (host(gx) * d).sum()) <= 1e-5 * np.abs(host(gx) * d).sum()
        d = rs.randn(dim)
        diff = (loss(hd, wd + step * d) - loss(hd, wd - step * d)) / (2 * step)
        assert abs(diff - (host(gw) * d).sum()) <= 1e-5 * np.abs(host(gw) * d).sum()


@pytest.mark.parametrize("dim", [100, 4096, 33000])
def test_backward_in_place_and_of_rows_that_lie_apart(dim):
    dt, rows = torch.bfloat16, 5
    h, w = normal(1, rows, dim, dtype=dt), normal(2, dim, dtype=dt)
    gy, gs = normal(3, rows, dim, dtype=dt), normal(4, rows, dim, dtype=dt)
    rstd = run_fwd(h, None, w, ("rstd",))["rstd"]
    want = run_bwd(h, w, rstd, gy, gs)
    for place in range(3):
        t = [h.clone(), gy.clone(), gs.clone()]
        ws = torch.empty(B.dsq_rms_norm_bwd_bytes(rows, dim), dtype=torch.uint8, device="cuda")
        gw = torch.empty(dim, device="cuda")
        B.dsq_rms_norm_bwd(t[0], w, rstd, t[1], t[2], t[place], gw, ws)
        assert torch.equal(t[place], want[0]) and torch.equal(gw, want[1])
    apart = lambda v: torch.cat([v, v[:, :8]], 1)[:, :dim]
    got = run_bwd(apart(h), w, rstd, apart(gy), apart(gs))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    one = gy[:1].expand(rows, dim)
    check_bwd(h, w, rstd, one, one, *run_bwd(h, w, rstd, one, one))


def test_no_rows():
    e = torch.empty(0, 64, device="cuda")
    B.dsq_rms_norm(e, None, None, EPS, e, None, None, None, None)
    gw = torch.full((64,), 3.0, device="cuda")
    B.dsq_rms_norm_bwd(e, None, torch.empty(0, device="cuda"), e, None, e, gw, None)
    assert not gw.any()


def test_more_than_2_31_elements():
    """Offsets past 32 bits: the last rows of a tensor of 2.2e9 elements."""
    rows, dim = 525000, 4096
    x = torch.empty(rows, dim, dtype=torch.bfloat16, device="cuda")
    tail = normal(1, 4, dim, dtype=torch.bfloat16)
    x[-4:] = tail
    x[:4] = tail
    w = normal(2, dim, dtype=torch.bfloat16)
    y = torch.empty_like(x)
    codes = torch.empty(rows, dim, dtype=torch.int8, device="cuda")
    scales = torch.empty(rows, device="cuda")
    B.dsq_rms_norm(x, None, w, EPS, None, y, codes, scales, None)
    small = run_fwd(tail, None, w)
    for at in (slice(0, 4), slice(rows - 4, rows)):
        assert torch.equal(y[at], small["y"]) and torch.equal(codes[at], small["codes"]) and torch.equal(scales[at], small["scales"])
