"""Norms of heads with the rotation in the same pass, the cache they write, and their backward pass, against float64."""
import numpy as np
import pytest
import torch

from heads_helpers import B, DTYPES, assert_within, check_rope, half_step, host, normal, oracle, qkv, rotation, tiny

pytestmark = pytest.mark.gpu
EPS = 1e-6


def forward(q, k, turning, interleaved=False, qw=None, kw=None, eps=EPS, q_out=None, k_out=None, cache=None, v=None):
    q_out = torch.empty(q.shape, dtype=q.dtype, device="cuda") if q_out is None else q_out
    if cache is None and k_out is None:
        k_out = torch.empty(k.shape, dtype=q.dtype, device="cuda")
    B.dsq_qk_norm_rope(q, k, v, qw, kw, eps, *turning, interleaved, q_out, k_out, *(cache or (None, None, None)))
    return q_out, k_out


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,hq,hk,dim,rope_dim,axes", [(1, 1, 1, 8, 0, 1), (3, 5, 1, 16, 16, 1), (2, 4, 2, 24, 16, 2), (7, 32, 8, 128, 128, 1),
                                                          (300, 6, 2, 80, 48, 3), (5, 3, 3, 64, 32, 1), (4, 2, 1, 256, 256, 16), (9, 40, 8, 200, 192, 2)])
def test_forward(rows, hq, hk, dim, rope_dim, axes, interleaved, dtype):
    dt = DTYPES[dtype]
    q, k, _ = qkv(rows + dim, rows, hq, hk, dim, dt)
    qw, kw = normal(1, dim, dtype=dt), normal(2, dim, dtype=dt)
    turning = rotation(rows, rows, rope_dim, axes)
    for weights, eps in (((qw, kw), EPS), ((None, kw), 0.5), ((None, None), 0.0)):
        outs = forward(q, k, turning, interleaved, *weights, eps)
        for x, w, got, what in zip((q, k), weights, outs, "qk"):
            check_rope(x, w, eps, turning, interleaved, got, what)


def test_far_positions_and_sizes():
    """Positions up to the ends of int32, heads of the largest and smallest numbers of their type, a head of zeros."""
    for dt in DTYPES.values():
        q, k, _ = qkv(3, 6, 4, 2, 64, dt)
        q, k = q.contiguous(), k.contiguous()
        q[0] *= 1e4
        q[1] = 0
        q[2] *= 2.0 ** -20
        if dt != torch.float16:
            q[3] *= 2.0 ** 100
        positions = torch.tensor([[2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 0, -1, 131071]], dtype=torch.int32, device="cuda")
        frequencies = torch.tensor(1e4 ** -(np.arange(32) / 32), dtype=torch.float32, device="cuda")
        outs = forward(q, k, (positions, None, frequencies), False, None, None, 1e-12)
        # (an angle of 2^31 in binary64 is off by 2^-23 of the products and the factor of pi, twice)
        angle = oracle.angles(host(positions).astype(np.int64), None, host(frequencies))
        for x, got in zip((q, k), outs):
            want, bound = oracle.norm_rope(host(x), None, 1e-12, angle, False)
            far = np.abs(angle).max(1)[:, None, None] * 2.0 ** -51
            bound = bound + far * oracle.mixed(want, angle, False) * 1.5
            assert_within(host(got), want, bound + half_step(dt) * (np.abs(want) + bound) + tiny(dt), str(dt))
        assert not outs[0][1].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", [1, 4, 64])
def test_cache(dtype, page):
    """Keys and values in their slots, with and without k_out; slots outside the cache and what no slot names stay as they are."""
    dt, rows, hq, hk, dim = DTYPES[dtype], 37, 6, 3, 40
    q, k, v = qkv(5, rows, hq, hk, dim, dt)
    turning = rotation(4, rows, 32)
    pages = 64 // page + 3
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(1))[:rows]
    slots[[3, 9, 11, 20]] = torch.tensor([-1, pages * page, 2 ** 62, -2 ** 63])
    slots = slots.cuda()
    q0, k0 = forward(q, k, turning)
    for with_k in (True, False):
        kc, vc = (torch.full((pages, hk, page, dim), 7.0, dtype=dt, device="cuda") for _ in range(2))
        k_out = torch.empty(k.shape, dtype=dt, device="cuda") if with_k else None
        q1, k1 = forward(q, k, turning, cache=(kc, vc, slots), v=v, k_out=k_out)
        assert torch.equal(q0, q1) and (not with_k or torch.equal(k0, k1))
        for cache, heads in ((kc, k0), (vc, v)):
            want = torch.full((pages * page, hk, dim), 7.0, dtype=dt, device="cuda")
            for r, s in enumerate(slots.tolist()):
                if 0 <= s < pages * page:
                    want[s] = heads[r]
            assert torch.equal(cache.transpose(1, 2).reshape(-1, hk, dim), want)


def test_values_go_to_the_cache_as_they_are():
    for dt, whole in ((torch.float16, torch.int16), (torch.bfloat16, torch.int16), (torch.float32, torch.int32)):
        bits = torch.randint(-2 ** 15, 2 ** 15, (64, 2, 16), dtype=torch.int64).to(whole).cuda()
        v = bits.view(dt)
        q, k, _ = qkv(6, 64, 2, 2, 16, dt)
        kc, vc = (torch.zeros(4, 2, 16, 16, dtype=dt, device="cuda") for _ in range(2))
        forward(q, k, rotation(2, 64, 16), cache=(kc, vc, torch.arange(64, device="cuda")), v=v)
        assert torch.equal(vc.view(whole).transpose(1, 2).reshape(64, 2, 16), bits)


def test_rows_and_heads_apart_and_in_place():
    for dt in DTYPES.values():
        q, k, _ = qkv(8, 9, 4, 2, 48, dt)
        turning = rotation(6, 9, 48)
        want = forward(q, k, turning)
        # heads before rows, and parts of a wider tensor whose rest is left alone
        room = torch.full((6, 9, 64), 5.0, dtype=dt, device="cuda")
        outs = room[:4, :, 8:56].transpose(0, 1), room[4:, :, 8:56].transpose(0, 1)
        forward(q, k, turning, q_out=outs[0], k_out=outs[1])
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
        assert (room[..., :8] == 5).all() and (room[..., 56:] == 5).all()
        # a row and a head that repeat
        got = forward(q[:1].expand(9, -1, -1), k[:, :1].expand(-1, 2, -1), turning)
        same = forward(q[:1].expand(9, -1, -1).contiguous(), k[:, :1].expand(-1, 2, -1).contiguous(), turning)
        assert all(torch.equal(a, b) for a, b in zip(got, same))
        whole = normal(8, 9, 8, 48, dtype=dt)
        forward(whole[:, :4], whole[:, 4:6], turning, q_out=whole[:, :4], k_out=whole[:, 4:6])
        assert torch.equal(whole[:, :4], want[0]) and torch.equal(whole[:, 4:6], want[1])


def test_one_kind_alone():
    q, k, _ = qkv(9, 5, 3, 2, 64, torch.bfloat16)
    turning = rotation(8, 5, 64)
    want = forward(q, k, turning)
    a, b = torch.empty_like(want[0]), torch.empty_like(want[1])
    B.dsq_qk_norm_rope(q, None, None, None, None, EPS, *turning, False, a, None, None, None, None)
    B.dsq_qk_norm_rope(None, k, None, None, None, EPS, *turning, False, None, b, None, None, None)
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])


def test_an_infinity_spoils_its_head_alone():
    q, k, _ = qkv(10, 6, 4, 2, 64, torch.float32)
    q = q.contiguous()
    turning = rotation(8, 6, 64)
    want = forward(q, k, turning)
    q[2, 1, 5], q[4, 0, 63] = float("inf"), float("nan")
    got = forward(q, k, turning)
    spoilt = torch.zeros(6, 4, dtype=torch.bool, device="cuda")
    spoilt[2, 1] = spoilt[4, 0] = True
    assert torch.equal(got[0][~spoilt], want[0][~spoilt]) and torch.equal(got[1], want[1])
    assert not torch.isfinite(got[0][spoilt]).all(-1).any()


# ---- backward -------------------------------------------------------------------------------------

def check_grads(x, weight, eps, turning, interleaved, grad, gx, gw, terms, what):
    angle = oracle.angles(host(turning[0]).astype(np.int64), None if turning[1] is None else turning[1].cpu().numpy(), host(turning[2]))
    want, bound, ww, size = oracle.norm_rope_grads(host(x), None if weight is None else host(weight), eps, angle, interleaved, host(grad))
    assert_within(host(gx), want, bound + half_step(x.dtype) * (np.abs(want) + bound) + tiny(x.dtype), what)
    if gw is not None:
        # a term is off by 12 half steps; sums of `terms` numbers in binary32, then binary64
        assert_within(host(gw), ww, (13 + terms) * oracle.U * size, what + " weight")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,hq,hk,dim,rope_dim,axes", [(1, 1, 1, 8, 0, 1), (3, 5, 1, 16, 16, 1), (7, 32, 8, 128, 128, 1), (2100, 6, 2, 80, 48, 3),
                                                          (1300, 3, 3, 64, 32, 1), (4, 2, 1, 256, 256, 2), (9, 40, 8, 200, 192, 2)])
def test_backward(rows, hq, hk, dim, rope_dim, axes, interleaved, dtype):
    dt = DTYPES[dtype]
    q, k, _ = qkv(rows + dim, rows, hq, hk, dim, dt)
    gq, gk, _ = qkv(rows + dim + 1, rows, hq, hk, dim, dt)
    qw, kw = normal(1, dim, dtype=dt), normal(2, dim, dtype=dt)
    turning = rotation(rows, rows, rope_dim, axes)
    size = B.dsq_qk_norm_rope_bwd_bytes(rows, hq, hk, dim)
    # (rows a workgroup takes, and its heads; a workgroup's sums are 2 dim numbers)
    terms = -(-rows // min(rows, size // (8 * dim))) * 16 + 256
    for weights, eps in (((qw, kw), EPS), ((None, None), 0.0)):
        out = [torch.empty(t.shape, dtype=dt, device="cuda") for t in (q, k)]
        gws = [torch.full((dim,), 9.0, device="cuda") if eps else None for _ in "qk"]
        ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") if eps else None
        for again in range(2):
            B.dsq_qk_norm_rope_bwd(q, k, *weights, eps, *turning, interleaved, gq, gk, *out, *gws, ws)
            now = [t.clone() for t in out + [g for g in gws if g is not None]]
            if again:
                assert all(torch.equal(a, b) for a, b in zip(now, first))          # the same bits every time
            first = now
        for x, w, g, o, gw, what in zip((q, k), weights, (gq, gk), out, gws, "qk"):
            check_grads(x, w, eps, turning, interleaved, g, o, gw, terms, what)


@pytest.mark.parametrize("dim,rows", [(8, 100), (16, 9), (32, 33), (256, 5)])
def test_backward_of_few_heads(dim, rows):
    """Several rows a workgroup, the last one not full; queries alone, one weight's gradient alone."""
    q, _, _ = qkv(20, rows, 1, 1, dim, torch.float32)
    g, w, turning = normal(21, rows, 1, dim), normal(22, dim), rotation(14, rows, dim // 16 * 16)
    gx, gw = torch.empty(rows, 1, dim, device="cuda"), torch.empty(dim, device="cuda")
    ws = torch.full((B.dsq_qk_norm_rope_bwd_bytes(rows, 1, 0, dim),), 0xFF, dtype=torch.uint8, device="cuda")
    B.dsq_qk_norm_rope_bwd(q, None, w, None, EPS, *turning, False, g, None, gx, None, gw, None, ws)
    check_grads(q, w, EPS, turning, False, g, gx, gw, rows + 256, "q")
    y = torch.empty_like(gx)
    B.dsq_qk_norm_rope(q, None, None, w, None, EPS, *turning, False, y, None, None, None, None)
    check_rope(q, w, EPS, turning, False, y, "q")


def test_backward_in_place_and_without_weights():
    q, k, _ = qkv(11, 12, 4, 2, 64, torch.float32)
    g, gk, _ = qkv(12, 12, 4, 2, 64, torch.float32)
    turning = rotation(10, 12, 64)
    want = [torch.empty(t.shape, device="cuda") for t in (q, k)]
    B.dsq_qk_norm_rope_bwd(q, k, None, None, EPS, *turning, False, g, gk, *want, None, None, None)
    over = [t.clone() for t in (g, gk)]
    B.dsq_qk_norm_rope_bwd(q, k, None, None, EPS, *turning, False, *over, *over, None, None, None)
    assert all(torch.equal(a, b) for a, b in zip(over, want))
    over = [t.contiguous().clone() for t in (q, k)]
    B.dsq_qk_norm_rope_bwd(*over, None, None, EPS, *turning, False, g, gk, *over, None, None, None)
    assert all(torch.equal(a, b) for a, b in zip(over, want))


def test_backward_against_differences():
    """Gradients against central differences of the float64 oracle: a step of 1e-6 leaves 1e-10 of each, binary32 arithmetic some 1e-6."""
    rows, hq, hk, dim = 5, 3, 2, 48
    q, k, _ = qkv(13, rows, hq, hk, dim, torch.float32)
    gq, gk, _ = qkv(14, rows, hq, hk, dim, torch.float32)
    qw, kw = normal(1, dim), normal(2, dim)
    turning = rotation(12, rows, 32, 2)
    out, gws = [torch.empty(t.shape, device="cuda") for t in (q, k)], [torch.empty(dim, device="cuda") for _ in "qk"]
    ws = torch.empty(B.dsq_qk_norm_rope_bwd_bytes(rows, hq, hk, dim), dtype=torch.uint8, device="cuda")
    B.dsq_qk_norm_rope_bwd(q, k, qw, kw, EPS, *turning, True, gq, gk, *out, *gws, ws)
    angle = oracle.angles(host(turning[0]).astype(np.int64), turning[1].cpu().numpy(), host(turning[2]))
    rs = np.random.RandomState(1)
    for x, w, g, gx, gw in ((q, qw, gq, out[0], gws[0]), (k, kw, gk, out[1], gws[1])):
        loss = lambda a, b: (host(g) * oracle.norm_rope(a, b, EPS, angle, True)[0]).sum()
        for at, got in ((0, gx), (1, gw)):
            for _ in range(3):
                d = rs.randn(*got.shape)
                up, down = [host(x), host(w)], [host(x), host(w)]
                up[at], down[at] = up[at] + 1e-6 * d, down[at] - 1e-6 * d
                diff = (loss(*up) - loss(*down)) / 2e-6
                assert abs(diff - (host(got) * d).sum()) <= 1e-5 * np.abs(host(got) * d).sum()


def test_no_rows():
    e = torch.empty(0, 2, 32, device="cuda", dtype=torch.float16)
    turning = rotation(2, 0, 32)
    B.dsq_qk_norm_rope(e, e, None, None, None, EPS, *turning, False, e, e, None, None, None)
    gw = torch.full((32,), 3.0, device="cuda")
    B.dsq_qk_norm_rope_bwd(e, e, None, None, EPS, *turning, False, e, e, e, e, gw, None, None)
    assert not gw.any()
