"""CPU-only checks of the calls for heads: sizes, refusals of the C interface before anything is launched, refusals of the binding, and
the oracle against itself."""
import numpy as np
import pytest
import torch

from oracle import heads as oracle
from paper_1908_05033_amd import binding as B

FAKE = 0x1000      # aligned, non-null; never dereferenced: validation fails first
INF, NAN = float("inf"), float("nan")


def test_sizes():
    n = [B.dsq_attention_bwd_bytes(*s) for s in ((1, 1), (1, 2), (100, 8), (5000, 8), (1 << 21, 8))]
    assert n == sorted(n) and n[0] >= 4 and n[-1] >= (1 << 24) * 4
    for bad in ((0, 1), (1, 0), ((1 << 21) + 1, 1), (1, 1025)):
        assert B.dsq_attention_bwd_bytes(*bad) == 0
    assert B.dsq_qk_norm_rope_bwd_bytes(1, 2, 1, 64) == 2 * 64 * 4
    for bad in ((0, 1, 1, 64), (1, 0, 0, 64), (1, -1, 1, 64), (1, 1, 1, 12), (1, 1, 1, 264), (1, 1025, 1, 64), ((1 << 21) + 1, 1, 1, 64)):
        assert B.dsq_qk_norm_rope_bwd_bytes(*bad) == 0
    # a workspace for more is never smaller
    for dim in (8, 64, 256):
        n = [B.dsq_qk_norm_rope_bwd_bytes(rows, 8, 2, dim) for rows in (1, 2, 300, 1024, 5000, 1 << 21)]
        assert n == sorted(n)
    n = [B.dsq_attention_cache_bytes(s, 1, 8, 2, 64) for s in (1, 2, 64, 1000, 65536)]
    assert n == sorted(n) and n[0] > 0
    for bad in ((0, 1, 8, 2, 64), (1, 0, 8, 2, 64), (1, 1, 8, 3, 64), (1, 1, 8, 2, 60), (1, 1, 8, 2, 136), (65537, 1, 8, 2, 64), (1, 1, 0, 2, 64),
                (1, 1, 2048, 2, 64)):
        assert B.dsq_attention_cache_bytes(*bad) == 0


def _rope(q=FAKE, qr=256, qh=64, k=FAKE, kr=128, kh=64, v=None, vr=128, vh=64, t=2, rows=4, hq=4, hk=2, dim=64, qw=None, kw=None, eps=1e-6, pos=FAKE, axes=1,
          pa=None, fr=FAKE, rd=64, il=0, qo=2 * FAKE, qor=256, qoh=64, ko=3 * FAKE, kor=128, koh=64, kc=None, vc=None, pages=4, page=16, slots=None):
    return B.load_library().dsq_qk_norm_rope(q, qr, qh, k, kr, kh, v, vr, vh, t, rows, hq, hk, dim, qw, kw, eps, pos, axes, pa, fr, rd, il, qo, qor, qoh, ko,
                                             kor, koh, kc, vc, pages, page, slots, None)


def _rope_bwd(q=FAKE, qr=256, qh=64, k=FAKE, kr=128, kh=64, t=2, rows=4, hq=4, hk=2, dim=64, qw=None, kw=None, eps=1e-6, pos=FAKE, axes=1, pa=None, fr=FAKE,
              rd=64, il=0, gqo=4 * FAKE, gqor=256, gqoh=64, gko=5 * FAKE, gkor=128, gkoh=64, gq=2 * FAKE, gqr=256, gqh=64, gk=3 * FAKE, gkr=128, gkh=64,
              gqw=None, gkw=None, ws=None, nbytes=0):
    return B.load_library().dsq_qk_norm_rope_bwd(q, qr, qh, k, kr, kh, t, rows, hq, hk, dim, qw, kw, eps, pos, axes, pa, fr, rd, il, gqo, gqor, gqoh, gko, gkor,
                                                 gkoh, gq, gqr, gqh, gk, gkr, gkh, gqw, gkw, ws, nbytes, None)


def test_rope_refusals():
    for f in (_rope, _rope_bwd):
        assert f(t=3) == 5 and f(t=-1) == 5
        assert f(rows=-1) == 4 and f(hq=-1) == 4 and f(hk=-1) == 4 and f(hq=0, hk=0) == 4 and f(dim=0) == 4 and f(rd=-16) == 4 and f(rd=80) == 4
        assert f(rows=(1 << 21) + 1) == 5 and f(hq=1025) == 5 and f(hk=1025) == 5 and f(dim=60, rd=0) == 5 and f(dim=264) == 5 and f(rd=24) == 5
        assert f(axes=0) == 5 and f(axes=17) == 5
        for eps in (-1e-6, INF, NAN):
            assert f(eps=eps) == 3
        assert f(eps=0.0, qw=FAKE) == 5 and f(eps=0.0, kw=FAKE) == 5
        assert f(q=None) == 1 and f(k=None) == 1 and f(pos=None) == 1 and f(fr=None) == 1
        for name in ("q", "k", "qw", "kw", "pos", "pa", "fr"):
            assert f(**{name: FAKE + 8}) == 6, name
        assert f(qr=-256) == 4 and f(kh=-64) == 4 and f(qr=260) == 6 and f(kh=68) == 6 and f(t=0, kh=66) == 6
        assert f(rows=0, q=None, k=None, pos=None) == 0 and f(rows=0, dim=12, rd=0) == 5
    assert _rope(qo=None) == 1 and _rope(ko=None) == 1
    assert _rope(qor=64) == 4 and _rope(qoh=32) == 4 and _rope(koh=0) == 4 and _rope(qor=64, qoh=248) == 4 and _rope(qoh=72) == 4
    assert _rope(qo=FAKE + 8) == 6 and _rope(ko=FAKE + 2) == 6
    assert _rope(qo=FAKE, qor=512) == 5 and _rope(ko=FAKE, koh=72, kor=144) == 5
    cache = dict(kc=4 * FAKE, vc=5 * FAKE, slots=FAKE, v=FAKE)
    for name in cache:
        assert _rope(**{**cache, name: None}) == 1, name
        assert _rope(**{**cache, name: FAKE + 8}) == 6, name
    assert _rope(**cache, pages=0) == 4 and _rope(**cache, pages=1 << 31) == 5 and _rope(**cache, vr=-1) == 4 and _rope(**cache, vr=132) == 6
    for page in (0, -1, 3, 48, 1 << 17):
        assert _rope(**cache, page=page) == 5
    assert _rope_bwd(gqo=None) == 1 and _rope_bwd(gk=None) == 1 and _rope_bwd(gqw=FAKE) == 1
    assert _rope_bwd(gqw=FAKE, ws=FAKE, nbytes=B.dsq_qk_norm_rope_bwd_bytes(4, 4, 2, 64) - 1) == 7
    assert _rope_bwd(eps=0.0, gkw=FAKE, ws=FAKE) == 5
    for name in ("gqo", "gko", "gq", "gk", "gqw", "gkw", "ws"):
        assert _rope_bwd(**{"ws": FAKE, name: FAKE + 4}) == 6, name
    assert _rope_bwd(gqr=64) == 4 and _rope_bwd(gkh=0) == 4 and _rope_bwd(gqor=-1) == 4 and _rope_bwd(gkoh=36) == 6
    assert _rope_bwd(gq=FAKE, gqr=512) == 5 and _rope_bwd(gk=5 * FAKE, gkr=256) == 5
    assert _rope_bwd(rows=0, gqw=FAKE + 4) == 6


def _attn(q=FAKE, qr=256, qh=64, k=FAKE, kr=128, kh=64, v=FAKE, vr=128, vh=64, t=2, rows=4, keys=4, hq=4, hk=2, dim=64, qs=None, ks=None, n=1, scale=1.0,
          out=2 * FAKE, outr=256, outh=64, lse=None):
    return B.load_library().dsq_attention(q, qr, qh, k, kr, kh, v, vr, vh, t, rows, keys, hq, hk, dim, qs, ks, n, 1, scale, out, outr, outh, lse, None)


def _attn_bwd(q=FAKE, qr=256, qh=64, k=FAKE, kr=128, kh=64, v=FAKE, vr=128, vh=64, out=FAKE, outr=256, outh=64, lse=FAKE, go=FAKE, gor=256, goh=64, t=2, rows=4,
              keys=4, hq=4, hk=2, dim=64, qs=None, ks=None, n=1, scale=1.0, gq=2 * FAKE, gqr=256, gqh=64, gk=3 * FAKE, gkr=128, gkh=64, gv=4 * FAKE, gvr=128,
              gvh=64, ws=FAKE, nbytes=1 << 20):
    return B.load_library().dsq_attention_bwd(q, qr, qh, k, kr, kh, v, vr, vh, out, outr, outh, lse, go, gor, goh, t, rows, keys, hq, hk, dim, qs, ks, n, 1, scale,
                                              gq, gqr, gqh, gk, gkr, gkh, gv, gvr, gvh, ws, nbytes, None)


def _cache(q=FAKE, qr=256, qh=64, t=2, rows=4, hq=4, hk=2, dim=64, qs=None, n=4, most=1, kc=FAKE, vc=FAKE, pages=8, page=16, table=FAKE, tr=4, tp=4, lengths=FAKE,
           tree=None, words=0, scale=1.0, out=2 * FAKE, outr=256, outh=64, ws=FAKE, nbytes=1 << 40):
    return B.load_library().dsq_attention_cache(q, qr, qh, t, rows, hq, hk, dim, qs, n, most, kc, vc, pages, page, table, tr, tp, lengths, tree, words, scale, out,
                                                outr, outh, ws, nbytes, None)


def test_attention_refusals():
    for f in (_attn, _attn_bwd, _cache):
        assert f(t=3) == 5 and f(rows=-1) == 4 and f(hq=0) == 4 and f(hk=0) == 4 and f(hk=3) == 4 and f(dim=0) == 4 and f(n=-1) == 4
        assert f(rows=(1 << 21) + 1) == 5 and f(hq=2048) == 5 and f(dim=60) == 5 and f(dim=136) == 5 and f(n=(1 << 16) + 1, qs=FAKE) == 5
        for scale in (0.0, -1.0, INF, NAN):
            assert f(scale=scale) == 3
        assert f(q=None) == 1 and f(out=None) == 1
        for name in ("q", "out", "qs"):
            assert f(**{name: FAKE + 8}) == 6, name
        assert f(qr=-8) == 4 and f(qh=68) == 6 and f(n=0, qs=FAKE, q=None) == 0
    for f in (_attn, _attn_bwd):
        assert f(keys=-1) == 4 and f(keys=(1 << 21) + 1) == 5 and f(n=2) == 4 and f(ks=FAKE) == 1 and f(qs=FAKE, ks=FAKE + 4) == 6
        assert f(k=None) == 1 and f(v=None) == 1 and f(k=FAKE + 8) == 6 and f(v=FAKE + 8) == 6 and f(kr=-1) == 4 and f(vh=4) == 6 and f(lse=FAKE + 4) == 6
    assert _attn(rows=0, q=None, out=None) == 0
    for f in (_attn, _cache):
        assert f(outr=64) == 4 and f(outh=0) == 4 and f(outr=252) == 4 and f(outr=260) == 6
    for name in ("lse", "go", "gq", "gk", "gv", "ws"):
        assert _attn_bwd(**{name: None}) == 1, name
        assert _attn_bwd(**{name: FAKE + 8}) == 6, name
    assert _attn_bwd(gqr=64) == 4 and _attn_bwd(gkh=0) == 4 and _attn_bwd(gvr=64) == 4 and _attn_bwd(goh=4) == 6 and _attn_bwd(outr=-8) == 4
    assert _attn_bwd(nbytes=63) == 7 and _attn_bwd(rows=0, keys=0, q=None) == 0
    assert _cache(most=0) == 4 and _cache(most=(1 << 21) + 1) == 5 and _cache(pages=-1) == 4 and _cache(tp=-1) == 4 and _cache(n=3) == 4
    assert _cache(tree=FAKE) == 4 and _cache(tree=FAKE + 8, words=1) == 6 and _cache(pages=1 << 31) == 5 and _cache(tr=-4) == 4
    for page in (0, -16, 24, 1 << 17):
        assert _cache(page=page) == 5
    assert _cache(tp=(1 << 14) + 1, page=1 << 16) == 5 and _cache(rows=1 << 16, n=1 << 16, tp=1 << 12, page=1 << 16) == 5
    assert _cache(most=1 << 21, hq=1024, hk=1, qr=65536, outr=65536, rows=1, n=1, tp=1) == 5
    assert _cache(rows=200, n=200, tp=1 << 14, page=1 << 16) == 5
    for name in ("kc", "vc", "table", "lengths", "ws"):
        assert _cache(**{name: None}) == 1, name
        assert _cache(**{name: FAKE + 8}) == 6, name
    assert _cache(nbytes=B.dsq_attention_cache_bytes(4, 1, 4, 2, 64) - 1) == 7
    assert _cache(rows=0, qs=FAKE, q=None) == 0


def test_refuses_launches_of_too_many_threads():
    """A launch has fewer than 2^32 threads.  (Without pointers: what is not refused for its size is for them, and nothing is launched.)"""
    apart = dict(qr=1024 * 64, outr=1024 * 64, hq=1024, hk=1024, kr=1024 * 64, vr=1024 * 64, q=None)
    for f in (_attn, _attn_bwd):
        for rows, keys, n, want in ((1 << 21, 4, 1, 5), (4, 1 << 21, 1, 5), (392960, 4, 1, 1), (4, 392960, 1, 1), (393216, 4, 1, 5), (4, 393216, 1, 5),
                                    (4, 4, 3000, 1), (4, 4, 3200, 5), (4, 4, 1 << 16, 5)):
            assert f(**apart, rows=rows, keys=keys, n=n, qs=FAKE) == want, (rows, keys, n)
    apart = dict(qr=1024 * 64, outr=1024 * 64, hq=1024, q=None)
    for rows, n, hk, want in ((1 << 16, 1 << 16, 8, 5), ((1 << 16) - 1, (1 << 16) - 1, 32, 1), (1 << 15, 1 << 15, 128, 5), ((1 << 15) - 1, (1 << 15) - 1, 128, 1)):
        assert _cache(**apart, rows=rows, n=n, hk=hk) == want, (rows, n, hk)
    assert _cache(**apart, rows=4, n=4, hk=8, most=1 << 21) == 5 and _cache(**apart, rows=4, n=1, hk=8, most=1 << 17, qs=FAKE) == 1


def test_binding_takes_device_tensors_alone():
    x, u8, i32 = torch.zeros(4, 2, 64), torch.zeros(1 << 16, dtype=torch.uint8), torch.zeros(5, dtype=torch.int32)
    c = torch.zeros(2, 2, 16, 64)
    for call in (lambda q: B.dsq_qk_norm_rope(q, x, None, None, None, 1e-6, None, None, None, False, x, x, None, None, None),
                 lambda q: B.dsq_qk_norm_rope_bwd(q, x, None, None, 1e-6, None, None, None, False, x, x, x, x, None, None, None),
                 lambda q: B.dsq_attention(q, x, x, None, None, True, 1.0, x, None),
                 lambda q: B.dsq_attention_bwd(q, x, x, x, x, x, None, None, True, 1.0, x, x, x, u8),
                 lambda q: B.dsq_attention_cache(q, None, 1, c, c, i32, i32, None, 1.0, x, u8)):
        with pytest.raises(TypeError):
            call(x)
    with pytest.raises(B.DsqError) as e:
        B.dsq_attention(None, x, x, None, None, True, 1.0, x, None)
    assert e.value.status == 1
    with pytest.raises(B.DsqError) as e:
        B.dsq_qk_norm_rope(None, None, None, None, None, 1e-6, None, None, None, False, None, None, None, None, None)
    assert e.value.status == 1


CALLS = {"qk_norm_rope": 16, "qk_norm_rope_bwd": 17, "attention": 10, "attention_bwd": 15, "attention_cache": 12}


@pytest.mark.parametrize("name", CALLS)
def test_native_marshalling_leaves_other_forms_alone(name):
    f, n = getattr(B.load_marshal(), name), CALLS[name]
    cpu = torch.zeros(4, 2, 64)
    for args in ([None] * n, [cpu] * n, [cpu] + [None] * (n - 1), [0x1000] * n, [1.0] * n, [object()] * n, [torch.zeros(4, 2, 64, device="meta")] * n):
        assert f(*args) is None
    assert f() is None and f(*[None] * (n + 1)) is None and f(*[None] * (n - 1)) is None
    for args in ((), (1,) * 4, (1,) * 6):
        with pytest.raises(TypeError):
            B.load_marshal().init_heads(*args)
    with pytest.raises(TypeError):
        B.load_marshal().init_heads(*["x"] * 5)


def test_oracle_gradients_are_the_formulas_differences():
    rs = np.random.RandomState(1)
    q, k, v, g = rs.randn(5, 8), rs.randn(7, 8), rs.randn(7, 8), rs.randn(5, 8)
    seen = oracle.causal(5, 7)
    r = oracle.attention(q, k, v, seen, 0.4, 0.0, g)
    loss = lambda a, b, c: (g * oracle.attention(a, b, c, seen, 0.4, 0.0)["out"][0]).sum()
    for i, name in enumerate(("dq", "dk", "dv")):
        x = [q, k, v]
        d = rs.randn(*x[i].shape)
        up, down = list(x), list(x)
        up[i], down[i] = x[i] + 1e-6 * d, x[i] - 1e-6 * d
        assert abs((loss(*up) - loss(*down)) / 2e-6 - (r[name][0] * d).sum()) < 1e-8
    angle, w = rs.randn(3, 4), rs.randn(8)
    x, g = rs.randn(3, 2, 8), rs.randn(3, 2, 8)
    for interleaved in (False, True):
        gx, _, gw, _ = oracle.norm_rope_grads(x, w, 1e-6, angle, interleaved, g)
        loss = lambda a, b: (g * oracle.norm_rope(a, b, 1e-6, angle, interleaved)[0]).sum()
        for got, at in ((gx, 0), (gw, 1)):
            d = rs.randn(*got.shape)
            up, down = [x, w], [x, w]
            up[at], down[at] = up[at] + 1e-6 * d, down[at] - 1e-6 * d
            assert abs((loss(*up) - loss(*down)) / 2e-6 - (got * d).sum()) < 1e-8


def test_oracle_tree_mask():
    words = np.array([[1, 0], [2, 0], [1 | 4, 0], [8, 1 << 3]], np.uint64)
    m = oracle.tree_mask(4, 6, words)
    assert m.tolist() == [[True, True, True, False, False, False], [True, True, False, True, False, False], [True, True, True, False, True, False],
                          [True, True, False, False, False, True]]
    assert (oracle.tree_mask(3, 2) == oracle.causal(3, 2)).all() and not oracle.causal(3, 2)[0].any()
    wide = np.zeros((70, 2), np.uint64)
    wide[69, 1] = 1 << 4
    assert np.flatnonzero(oracle.tree_mask(70, 75, wide)[69]).tolist() == [0, 1, 2, 3, 4, 5 + 68]
