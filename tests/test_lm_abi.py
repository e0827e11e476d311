"""CPU-only checks of the language-model calls: sizes, refusals of the C interface before anything is launched, and
refusals of the binding."""
import pytest
import torch

from paper_1908_05033_amd import binding as B

FAKE = 0x1000      # aligned, non-null; never dereferenced: validation fails first
INF, NAN = float("inf"), float("nan")


def test_sizes():
    assert [B.dsq_code_row_bytes(d) for d in (1, 128, 129, 4096, 0, -1, (1 << 20) + 1)] == [128, 128, 256, 4096, 0, 0, 0]
    assert B.dsq_w4_packed_bytes(1, 1) == 128 * 64 and B.dsq_w4_packed_bytes(4096, 4100) == 4096 * 4224 // 2
    assert B.dsq_w4_scale_bytes(1000, 300, 64) == 1024 * 6 * 4 and B.dsq_w4_scale_bytes(16, 128, 32) == 128 * 4 * 4
    for bad in ((0, 1), (1, 0), ((1 << 24) + 1, 1), (1, (1 << 20) + 1), (1 << 24, 1 << 20)):
        assert B.dsq_w4_packed_bytes(*bad) == 0 and B.dsq_w4_scale_bytes(*bad, 128) == 0
    assert B.dsq_w4_scale_bytes(16, 128, 48) == 0 and B.dsq_w4_scale_bytes(16, 128, 0) == 0
    assert B.dsq_rms_norm_bwd_bytes(1, 4096) == 4096 * 4
    assert B.dsq_rms_norm_bwd_bytes(1 << 20, 4096) % (4096 * 4) == 0
    assert B.dsq_rms_norm_bwd_bytes(0, 64) == 0 and B.dsq_rms_norm_bwd_bytes(64, 0) == 0
    # a workspace for more rows is never smaller
    for dim in (1, 100, 600, 5000, 40000):
        n = [B.dsq_rms_norm_bwd_bytes(rows, dim) for rows in (1, 2, 16, 17, 500, 513, 8192, 1 << 21)]
        assert n == sorted(n)


def _norm(x=FAKE, xs=64, res=None, rs=64, w=None, t=2, rows=4, dim=64, eps=1e-6, s=None, y=FAKE, codes=None, nbytes=1 << 20,
          scales=None, rstd=None):
    return B.load_library().dsq_rms_norm(x, xs, res, rs, w, t, rows, dim, eps, s, y, codes, nbytes, scales, rstd, None)


def test_rms_norm_refusals():
    assert _norm(t=3) == 5 and _norm(t=-1) == 5
    assert _norm(rows=-1) == 4 and _norm(dim=0) == 4 and _norm(dim=-3) == 4
    assert _norm(rows=(1 << 21) + 1) == 5 and _norm(dim=(1 << 20) + 1) == 5
    for eps in (0.0, -1e-6, INF, NAN):
        assert _norm(eps=eps) == 3
    assert _norm(x=None) == 1 and _norm(y=None) == 1
    assert _norm(codes=FAKE) == 1 and _norm(scales=FAKE) == 1
    assert _norm(xs=-64) == 4 and _norm(res=FAKE, rs=-1) == 4
    for k in ("x", "res", "w", "s", "y", "rstd"):
        assert _norm(**{k: FAKE + 8}) == 6, k
    assert _norm(codes=FAKE + 4, scales=FAKE) == 6 and _norm(codes=FAKE, scales=FAKE + 4) == 6
    assert _norm(codes=FAKE, scales=FAKE, nbytes=4 * 128 - 1) == 7
    assert _norm(x=FAKE, xs=72, y=FAKE) == 5 and _norm(res=2 * FAKE, rs=0, s=2 * FAKE) == 5
    assert _norm(rows=0, x=None, y=None) == 0                      # no rows: nothing to do
    assert _norm(rows=0, eps=0.0) == 3 and _norm(rows=0, dim=0) == 4


def _bwd(h=FAKE, hs=64, w=None, r=FAKE, gy=FAKE, gys=64, gs=None, gss=64, t=2, rows=4, dim=64, gx=2 * FAKE, gw=None, ws=None,
         nbytes=0):
    return B.load_library().dsq_rms_norm_bwd(h, hs, w, r, gy, gys, gs, gss, t, rows, dim, gx, gw, ws, nbytes, None)


def test_rms_norm_bwd_refusals():
    assert _bwd(t=7) == 5 and _bwd(rows=-1) == 4 and _bwd(dim=0) == 4
    assert _bwd(rows=(1 << 21) + 1) == 5 and _bwd(dim=(1 << 20) + 1) == 5
    for k in ("h", "r", "gy", "gx"):
        assert _bwd(**{k: None}) == 1, k
        assert _bwd(**{k: FAKE + 4}) == 6, k
    assert _bwd(gw=FAKE) == 1
    assert _bwd(hs=-1) == 4 and _bwd(gys=-1) == 4 and _bwd(gs=FAKE, gss=-1) == 4
    need = B.dsq_rms_norm_bwd_bytes(4, 64)
    assert need > 0 and _bwd(gw=FAKE, ws=FAKE, nbytes=need - 1) == 7
    assert _bwd(gw=FAKE, ws=FAKE + 8, nbytes=need) == 6 and _bwd(gw=FAKE + 4, ws=FAKE, nbytes=need) == 6
    assert _bwd(gx=FAKE, hs=72) == 5 and _bwd(gs=2 * FAKE, gss=0) == 5
    assert _bwd(rows=0, h=None, r=None, gy=None, gx=None) == 0
    assert _bwd(rows=0, gw=FAKE + 4) == 6


def _pack(w=FAKE, codes=None, scale=None, zero=None, N=16, K=128, group=64, wp=FAKE, wn=1 << 20, sp=FAKE, sn=1 << 20):
    return B.load_library().dsq_pack_weights_w4(w, codes, scale, zero, N, K, group, wp, wn, sp, sn, None)


def test_pack_refusals():
    assert _pack(w=None) == 1 and _pack(wp=None) == 1 and _pack(sp=None) == 1
    assert _pack(w=None, codes=FAKE) == 1 and _pack(scale=FAKE) == 1 and _pack(zero=FAKE) == 1
    assert _pack(codes=FAKE, scale=FAKE, zero=FAKE) == 5          # both weights and codes
    assert _pack(N=0) == 4 and _pack(K=-1) == 4
    assert _pack(group=16) == 5 and _pack(group=0) == 5 and _pack(group=256) == 5 and _pack(K=(1 << 20) + 1) == 5
    assert _pack(w=FAKE + 4) == 6 and _pack(wp=FAKE + 4) == 6 and _pack(sp=FAKE + 8) == 6
    assert _pack(wn=128 * 64 - 1) == 7 and _pack(sn=128 * 2 * 4 - 1) == 7


def _lin(x=FAKE, xs=128, t=2, M=4, N=16, K=128, group=64, w=FAKE, s=FAKE, bias=None, out=FAKE, os=16):
    return B.load_library().dsq_linear_w4(x, xs, t, M, N, K, group, w, s, bias, out, os, None)


def _lin8(q=FAKE, nbytes=1 << 20, qs=FAKE, t=2, M=4, N=16, K=128, group=64, w=FAKE, s=FAKE, bias=None, out=FAKE, os=16):
    return B.load_library().dsq_linear_w4a8(q, nbytes, qs, M, N, K, group, w, s, bias, t, out, os, None)


def test_linear_refusals():
    for f in (_lin, _lin8):
        assert f(t=3) == 5 and f(group=65) == 5 and f(M=(1 << 21) + 1) == 5 and f(N=(1 << 24) + 1) == 5
        assert f(M=-1) == 4 and f(N=0) == 4 and f(K=0) == 4 and f(os=15) == 4
        for k in ("w", "s", "out"):
            assert f(**{k: None}) == 1, k
            assert f(**{k: FAKE + 8}) == 6, k
        assert f(bias=FAKE + 2) == 6
        assert f(M=0, w=None, out=None) == 0
    assert _lin(x=None) == 1 and _lin(x=FAKE + 2) == 6 and _lin(xs=-1) == 4
    assert _lin8(q=None) == 1 and _lin8(qs=None) == 1 and _lin8(q=FAKE + 1) == 6 and _lin8(qs=FAKE + 4) == 6
    assert _lin8(nbytes=4 * 128 - 1) == 7


def test_binding_takes_device_tensors_alone():
    x = torch.zeros(4, 64)
    u8 = torch.zeros(1 << 16, dtype=torch.uint8)
    for call in (lambda: B.dsq_rms_norm(x, None, None, 1e-6, None, x, None, None, None),
                 lambda: B.dsq_rms_norm_bwd(x, None, x, x, None, x, None, None),
                 lambda: B.dsq_pack_weights_w4(x, None, None, None, 4, 64, 64, u8, u8),
                 lambda: B.dsq_linear_w4(x, u8, u8, 16, 64, 64, None, x),
                 lambda: B.dsq_linear_w4a8(u8, x, u8, u8, 16, 64, 64, None, x)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(B.DsqError) as e:
        B.dsq_linear_w4(None, u8, u8, 16, 64, 64, None, x)
    assert e.value.status == 1
