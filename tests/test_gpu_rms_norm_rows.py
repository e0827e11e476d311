"""Rows of the norm at the edges of its kernels: in place, beside memory full of NaN, and far apart.  Tolerances as derived in
test_gpu_rms_norm.py."""
import pytest
import torch

from paper_1908_05033_amd import binding as B
from lm_helpers import DTYPES, host, normal
from test_gpu_rms_norm import EPS, check_bwd, check_fwd, run_bwd, run_fwd

pytestmark = pytest.mark.gpu
# one vector a thread, several, rows past the registers; whole vectors and odd ends
DIMS = [5, 250, 2048, 4591, 5120, 8191, 9001, 12288, 16383, 16500]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", DIMS)
def test_in_place(dim, dtype):
    dt, rows = DTYPES[dtype], 300
    x, res, w = normal(1, rows, dim, dtype=dt), normal(2, rows, dim, dtype=dt), normal(3, dim, dtype=dt)
    want = run_fwd(x, res, w)
    a, b = x.clone(), res.clone()
    B.dsq_rms_norm(a, b, w, EPS, b, a, None, None, None)
    assert torch.equal(b, want["sum"]) and torch.equal(a, want["y"])
    gy, gs = normal(4, rows, dim, dtype=dt), normal(5, rows, dim, dtype=dt)
    gx, gw = run_bwd(want["sum"], w, want["rstd"], gy, gs)
    for place in range(3):
        t = [want["sum"].clone(), gy.clone(), gs.clone()]
        ws = torch.empty(B.dsq_rms_norm_bwd_bytes(rows, dim), dtype=torch.uint8, device="cuda")
        got = torch.empty(dim, device="cuda")
        B.dsq_rms_norm_bwd(t[0], w, want["rstd"], t[1], t[2], t[place], got, ws)
        assert torch.equal(t[place], gx) and torch.equal(got, gw)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", DIMS)
def test_beside_memory_full_of_nan(dim, dtype):
    dt, rows = DTYPES[dtype], 19

    def inside(v):
        wide = torch.full((rows + 3, dim + 13), float("nan"), dtype=dt, device="cuda")
        wide[:rows, :dim] = v
        return wide[:rows, :dim]

    x, res, w = normal(1, rows, dim, dtype=dt), normal(2, rows, dim, dtype=dt), torch.full((dim + 40,), float("nan"), dtype=dt, device="cuda")
    w[:dim] = normal(3, dim, dtype=dt)
    w = w[:dim]
    out = run_fwd(inside(x), inside(res), w)
    check_fwd(x, res, w, out)
    gy, gs = normal(4, rows, dim, dtype=dt), normal(5, rows, dim, dtype=dt)
    gx, gw = run_bwd(inside(out["sum"]), w, out["rstd"], inside(gy), inside(gs))
    check_bwd(out["sum"], w, out["rstd"], gy, gs, gx, gw)


@pytest.mark.parametrize("dim", [251, 4591, 9001])
def test_outputs_end_with_their_rows(dim):
    """What lies behind the last row of each output stays as it was."""
    rows, dt = 33, torch.bfloat16
    x, w = normal(1, rows, dim, dtype=dt), normal(2, dim, dtype=dt)
    pitch = B.dsq_code_row_bytes(dim)
    room = lambda n, d: torch.full((n + 1000,), 7, dtype=d, device="cuda")
    s, y, q, qs, r = room(rows * dim, dt), room(rows * dim, dt), room(rows * pitch, torch.int8), room(rows, torch.float32), room(rows, torch.float32)
    B.dsq_rms_norm(x, None, w, EPS, s[:rows * dim].view(rows, dim), y[:rows * dim].view(rows, dim), q[:rows * pitch].view(rows, pitch), qs[:rows], r[:rows])
    gx, gw, n = room(rows * dim, dt), room(dim, torch.float32), B.dsq_rms_norm_bwd_bytes(rows, dim)
    ws = room(n, torch.uint8)
    B.dsq_rms_norm_bwd(x, w, r[:rows], x, None, gx[:rows * dim].view(rows, dim), gw[:dim], ws[:n])
    torch.cuda.synchronize()
    for t, used in ((s, rows * dim), (y, rows * dim), (q, rows * pitch), (qs, rows), (r, rows), (gx, rows * dim), (gw, dim), (ws, n)):
        assert (t[used:] == 7).all()


def test_rows_more_than_2_32_bytes_apart():
    rows, dim, far = 40, 1001, 125_000_003
    dt = torch.bfloat16
    big = torch.empty((rows - 1) * far + 4096, dtype=dt, device="cuda")
    x, gy = big.as_strided((rows, dim), (far, 1)), big.as_strided((rows, dim), (far, 1), 2048)
    x.copy_(normal(1, rows, dim, dtype=dt))
    gy.copy_(normal(2, rows, dim, dtype=dt))
    w = normal(3, dim, dtype=dt)
    out = run_fwd(x, None, w)
    check_fwd(x.contiguous(), None, w, out)
    gx, gw = run_bwd(x, w, out["rstd"], gy, x)
    check_bwd(x.contiguous(), w, out["rstd"], gy.contiguous(), x.contiguous(), gx, gw)
    assert host(gx).shape == (rows, dim)
