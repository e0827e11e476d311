"""Attention in float16 where one key has nearly all of the probability and its value is zero: the result is the sum of the small
probabilities of the others, which binary16 does not hold by itself (below 2^-14 with fewer digits, at 2^-25 not at all)."""
import numpy as np
import pytest
import torch

from heads_helpers import B, assert_within, half_step, host, oracle, starts, tiny
from test_gpu_attention import Call
from test_gpu_attention_cache import Case

pytestmark = pytest.mark.gpu
F16 = torch.float16
HALF = half_step(F16)
# A rounded operand is off by half a step, or by half the distance 2^-24 of the smallest numbers where it has fewer digits: with probabilities
# taken times 2^13, relative to the largest of their row, by 2^-25 - 13 of it.  Their sum is at least the largest.
LOST = 2.0 ** -38


def sunk(seed, rows, keys, hq, hk, dim, above):
    """Queries, keys and values [.., heads, dim] of which key 0 has a score `above` (natural logarithm) the others', which lie within 0.3, and no value."""
    rs = np.random.RandomState(seed)
    q, k, v = rs.randn(rows, hq, dim) * 0.1, rs.randn(keys, hk, dim) * 0.1, 1 + 0.5 * rs.rand(keys, hk, dim)
    q[..., 0], k[..., 0], k[0], v[0] = 8, 0, 0, 0
    k[0, :, 0] = above * dim ** 0.5 / 8
    return [torch.tensor(t, dtype=F16, device="cuda") for t in (q, k, v)]


def check(q, k, v, seen, out, lse, what):
    """One head."""
    r = oracle.attention(host(q), host(k), host(v), seen, q.shape[1] ** -0.5, HALF, tiny=LOST)
    want, bound = r["out"]
    # (the values are of one sign: the result is as large as the sum of its terms)
    assert (bound < 0.02 * np.abs(want) + 1e-7).all()
    assert_within(host(out), want, bound + HALF * (np.abs(want) + bound) + tiny(F16), what)
    if lse is not None:
        assert_within(host(lse), *r["lse"], what + " lse")


@pytest.mark.parametrize("above", [8.0, 12.0, 17.5, 18.5])
@pytest.mark.parametrize("keys,dim", [(33, 64), (1000, 64), (5000, 128), (5000, 80)])
def test_prompt(keys, dim, above):
    q, k, v = sunk(1, 40, keys, 4, 2, dim, above)
    c = Call(q, k, v, None, None, causal=False).forward()
    for h in (0, 3):
        check(q[:, h], k[:, h // 2], v[:, h // 2], np.ones((40, keys), bool), c.out[:, h], c.lse[h], "head %d" % h)


@pytest.mark.parametrize("dim", [64, 96, 128])
def test_prompt_of_many_rows(dim):
    """128 rows a workgroup: rows times heads are past the limit of the other kernel."""
    q, k, v = sunk(2, 1100, 1100, 48, 12, dim, 17.5)
    c = Call(q, k, v, None, None).forward()
    for h in (0, 47):
        check(q[:, h], k[:, h // 4], v[:, h // 4], oracle.causal(1100, 1100), c.out[:, h], c.lse[h], "head %d" % h)


@pytest.mark.parametrize("above", [12.0, 17.5, 18.5])
@pytest.mark.parametrize("lengths,drafted,heads", [([500, 100], [1, 1], (4, 2)), ([9000, 700], [1, 1], (4, 2)), ([9000, 700], [20, 33], (8, 2))])
def test_cache(lengths, drafted, heads, above):
    """One chunk, chunks that are joined, tiles."""
    hq, hk = heads
    c = Case(3, "f16", lengths, drafted, hq, hk, 64, 16)
    at = 0
    for s, (m, n) in enumerate(zip(lengths, drafted)):
        q, k, v = sunk(s, n, m, hq, hk, 64, above)
        c.q[at:at + n] = q
        at += n
        place = torch.arange(m, device="cuda")
        for cache, heads_of in zip(c.cache, (k, v)):
            cache[c.table[s].long()[place // 16], :, place % 16] = heads_of
        c.kv[s] = (k, v)
    c.run()
    at = 0
    for s, (m, n) in enumerate(zip(lengths, drafted)):
        for h in (0, hq - 1):
            k, v = (t[:, h // (hq // hk)] for t in c.kv[s])
            check(c.q[at:at + n, h], k, v, oracle.tree_mask(n, m), c.out[at:at + n, h], None, "sequence %d head %d" % (s, h))
        at += n
