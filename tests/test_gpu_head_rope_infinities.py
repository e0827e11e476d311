"""Norms of heads that hold an infinity or a NaN: the root of an infinite mean has the reciprocal 0, so finite elements become 0."""
import numpy as np
import pytest
import torch

from heads_helpers import B, DTYPES, host, normal, oracle, qkv, rotation

pytestmark = pytest.mark.gpu
EPS, INF, NAN = 1e-6, float("inf"), float("nan")
ROWS, HQ, HK, DIM, ROPE = 6, 4, 2, 80, 48
# (row, head, element): one of a pair, its second one, behind the rotated ones, two in one head
PLACES = [((0, 1, 5),), ((1, 0, 40),), ((2, 3, 70),), ((3, 2, 3), (3, 2, 77))]


def inputs(dtype):
    dt = DTYPES[dtype]
    q, k, _ = qkv(1, ROWS, HQ, HK, DIM, dt)
    return q.contiguous(), k.contiguous(), normal(2, DIM, dtype=dt), normal(3, DIM, dtype=dt), rotation(4, ROWS, ROPE)


def angle_of(turning):
    return oracle.angles(host(turning[0]).astype(np.int64), None, host(turning[2]))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("bad", [INF, -INF, NAN])
def test_forward(bad, interleaved, dtype):
    q, k, qw, kw, turning = inputs(dtype)
    run = lambda x: [B.dsq_qk_norm_rope(x, k, None, qw, kw, EPS, *turning, interleaved, *out, None, None, None) or out
                     for out in [(torch.full_like(q, 7), torch.full_like(k, 7))]][0]
    clean = run(q)
    x, spoilt = q.clone(), torch.zeros(ROWS, HQ, dtype=torch.bool, device="cuda")
    for places in PLACES:
        for at in places:
            x[at] = bad
            spoilt[at[:2]] = True
    got = run(x)
    assert torch.equal(got[0][~spoilt], clean[0][~spoilt]) and torch.equal(got[1], clean[1])
    with np.errstate(invalid="ignore"):
        want = oracle.norm_rope(host(x), host(qw), EPS, angle_of(turning), interleaved)[0]
    mine = host(got[0])[spoilt.cpu().numpy()]
    want = want[spoilt.cpu().numpy()]
    # (nothing but NaN and 0 in these heads, so there is nothing to round)
    assert np.array_equal(mine, want, equal_nan=True)
    if bad is NAN:
        assert np.isnan(mine).all()
    else:
        assert (np.isnan(mine).sum(1) <= 4).all() and (mine[~np.isnan(mine)] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_backward(dtype):
    """The head's own gradient is NaN, and of the weight's gradient the element of the infinity."""
    q, k, qw, kw, turning = inputs(dtype)
    gq, gk, _ = qkv(5, ROWS, HQ, HK, DIM, q.dtype)
    ws = torch.full((B.dsq_qk_norm_rope_bwd_bytes(ROWS, HQ, HK, DIM),), 0xFF, dtype=torch.uint8, device="cuda")

    def run(x):
        out = [torch.full_like(q, 7), torch.full_like(k, 7), torch.full((DIM,), 9.0, device="cuda"), torch.full((DIM,), 9.0, device="cuda")]
        B.dsq_qk_norm_rope_bwd(x, k, qw, kw, EPS, *turning, False, gq, gk, *out, ws)
        return out

    clean = run(q)
    x = q.clone()
    x[2, 1, 7] = INF
    without = q.clone()
    without[2, 1] = 0                                  # (a head of zeros adds nothing to the weight's gradient)
    got, rest = run(x), run(without)
    spoilt = torch.zeros(ROWS, HQ, dtype=torch.bool, device="cuda")
    spoilt[2, 1] = True
    assert torch.isnan(got[0][spoilt]).all() and torch.equal(got[0][~spoilt], clean[0][~spoilt])
    assert torch.equal(got[1], clean[1]) and torch.equal(got[3], clean[3])
    others = torch.arange(DIM, device="cuda") != 7
    assert torch.isnan(got[2][7]) and torch.equal(got[2][others], rest[2][others])
