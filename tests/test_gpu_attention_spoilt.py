"""Attention where values that rows see are infinite or NaN, beside others that they do not see: every element is what its own visible keys make of it, and a
call takes about as long as without them."""
import numpy as np
import pytest
import torch

from heads_helpers import B, DTYPES, assert_within, half_step, host, normal, oracle, operand_tiny, qkv, starts, tiny
from test_gpu_attention import Call
from test_gpu_attention_cache import Case

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
# rows, query heads, key heads: waves that split the keys, and 128 rows a workgroup
KINDS = {"few": (200, 4, 2), "many": (1100, 48, 4)}


def expected(q, k, v, seen, scale, dt):
    """(result, bound) of one head; infinities and NaN of the values that a row sees take the place of its finite part, without a bound."""
    finite = np.isfinite(v)
    r = oracle.attention(q, k, np.where(finite, v, 0), seen, scale, half_step(dt), tiny=operand_tiny(dt))
    want, bound = r["out"]
    bound = bound + half_step(dt) * (np.abs(want) + bound) + tiny(dt)
    with np.errstate(invalid="ignore"):
        for j, e in np.argwhere(~finite):
            want[seen[:, j], e] += v[j, e]
    return want, bound


def check(got, want, bound, what):
    odd = ~np.isfinite(want)
    assert np.array_equal(got[odd], want[odd], equal_nan=True), what
    assert_within(got[~odd], want[~odd], bound[~odd], what)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [40, 64, 80, 96, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind", KINDS)
def test_prompt(kind, causal, dim, dtype):
    """Infinities of one sign and of both early on, NaN in one element, NaN in all of a later key, which earlier rows share a tile with."""
    n, hq, hk = KINDS[kind]
    dt = DTYPES[dtype]
    q, k, v = qkv(dim, n, hq, hk, dim, dt)
    v = v.contiguous()
    v[3, 0, 5], v[40, 0, 7], v[3, 0, 7], v[50, 0, dim - 1] = INF, -INF, INF, NAN
    v[70, 0] = NAN
    v[n - 1, 1, 0] = -INF
    v[:, 1, 8], v[2::9, 1, 9], v[5::7, 1, 10] = INF, -INF, torch.tensor([INF, -INF] * n, dtype=dt, device="cuda")[:len(v[5::7])]
    c = Call(q, k, v, None, None, causal).forward()
    seen = oracle.causal(n, n) if causal else np.ones((n, n), bool)
    for h in (0, hq // hk - 1, hq // hk):
        kv = h // (hq // hk)
        want, bound = expected(host(q)[:, h], host(k)[:, kv], host(v)[:, kv], seen, c.scale, dt)
        check(host(c.out)[:, h], want, bound, "head %d" % h)
        r = oracle.attention(host(q)[:, h], host(k)[:, kv], np.zeros((n, dim)), seen, c.scale, 0.0)
        assert_within(host(c.lse)[h], *r["lse"], "lse")
    # other key heads are as without
    clean = Call(q, k, torch.where(torch.isfinite(v), v, 0), None, None, causal).forward()
    assert torch.equal(c.out[:, 2 * hq // hk:], clean.out[:, 2 * hq // hk:]) and torch.equal(c.lse[2 * hq // hk:], clean.lse[2 * hq // hk:])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [40, 64, 80, 96, 104, 128])
@pytest.mark.parametrize("kind", KINDS)
def test_keys_of_no_weight(kind, dim, dtype):
    """A key of minus infinity against queries that are positive there has a probability of zero, also where heads are narrower than their kernel's."""
    n, hq, hk = KINDS[kind]
    dt = DTYPES[dtype]
    q, k, v = (t.contiguous() for t in qkv(1, n, hq, hk, dim, dt))
    q[..., 0] = 1
    k[20, :, 0] = -INF
    k[0, :, 0] = 4                                         # (no row sees the key of no weight alone)
    c = Call(q, k, v, None, None).forward()
    seen = oracle.causal(n, n)
    seen[:, 20] = False
    without = host(k)
    without[20] = 0
    for h in (0, hq - 1):
        kv = h // (hq // hk)
        want, bound = expected(host(q)[:, h], without[:, kv], host(v)[:, kv], seen, c.scale, dt)
        check(host(c.out)[:, h], want, bound, "head %d" % h)
    # plus infinity, and NaN in a query or a key: the rows that have one are NaN, the others are not
    k[20, :, 0] = INF
    q[10, :, 3] = NAN
    k[60, :, 1] = NAN
    c.forward()
    rows = torch.zeros(n, dtype=torch.bool, device="cuda")
    rows[20:] = rows[10] = True
    assert torch.isnan(c.out[rows]).all() and torch.isnan(c.lse[:, rows]).all()
    assert torch.isfinite(c.out[~rows]).all() and torch.isfinite(c.lse[:, ~rows]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_near_the_end_of_their_type(dtype):
    """Sums of finite values that pass binary32 on the way, in many rows and over a cache, beside an infinity."""
    dt = DTYPES[dtype]
    q, k, _ = qkv(8, 1100, 48, 4, 64, dt)
    v = torch.full((1100, 4, 64), 3e38, dtype=dt, device="cuda")
    v[2, 0, 9] = INF
    c = Call(q, k, v, None, None).forward()
    part = c.out.double() / float(v[0, 0, 0])
    part[2:, :12, 9] = torch.where(torch.isposinf(part[2:, :12, 9]), 1.0, NAN)
    assert ((part - 1).abs() < 4 * half_step(dt) + 1100 * oracle.U).all()
    c = Case(9, dtype, [700, 90], [1, 1], 4, 2, 64, 16)
    c.cache[1].copy_(torch.where(torch.isnan(c.cache[1]), c.cache[1], 3e38))
    c.run()
    assert ((c.out.double() / float(v[0, 0, 0]) - 1).abs() < 4 * half_step(dt) + 5000 * oracle.U).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lengths,drafted,heads", [([300, 45], [12, 5], (4, 2)), ([5000, 700], [6, 3], (4, 2)), ([5000, 700, 90], [40, 17, 33], (8, 2))])
@pytest.mark.parametrize("dim", [40, 64, 128])
def test_cache(dim, lengths, drafted, heads, dtype):
    """Infinities in values before the drafted tokens and in drafted ones, NaN in drafted ones that some rows see, in one launch, chunks and tiles."""
    hq, hk = heads
    c = Case(7, dtype, lengths, drafted, hq, hk, dim, 16, tree=True)

    def put(which, s, j, kv, e, x):
        c.cache[which][int(c.table[s, j // 16]), kv, j % 16, e] = x
        c.kv[s][which][j, kv, e] = x

    n, m = lengths[0], drafted[0]
    put(1, 0, 2, 0, 5, INF)
    put(1, 0, n - m - 1, 0, 6, -INF)
    put(1, 0, n - m - 1, 0, 5, INF)
    put(1, 0, n - m + 1, 0, slice(None), NAN)
    for j in range(n):
        put(1, 0, j, 1, 7, INF)
    put(1, 1, 1, 1, 0, INF)
    put(1, 1, 0, 1, 0, -INF)
    c.run()
    at = 0
    for s, (n, m) in enumerate(zip(lengths, drafted)):
        seen = oracle.tree_mask(m, n, c.words[s])
        for h in range(hq):
            kv = h // (hq // hk)
            k, v = (host(t)[:, kv] for t in c.kv[s])
            check(host(c.out)[at:at + m, h], *expected(host(c.q)[at:at + m, h], k, v, seen, c.scale, c.dt), "sequence %d head %d" % (s, h))
        at += m


def took(run, n=5):
    """The least time of a call, ms."""
    run()
    times = []
    for _ in range(n):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in "ab")
        a.record()
        run()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b))
    return min(times)


@pytest.mark.parametrize("rows,heads,dim", [(2048, 8, 128), (2048, 8, 80), (4096, 16, 64), (4096, 16, 128)])
def test_time_of_a_prompt(rows, heads, dim):
    """A bad value that every later row sees costs no walk over the keys for each of them (which takes 38 ms and more; a busy card or clock is allowed for)."""
    q, k, v = (t.contiguous() for t in qkv(2, rows, heads, heads // 4, dim, torch.bfloat16))
    clean = took(Call(q, k, v, None, None).forward)
    for which, at, bad in ((1, (0, slice(None), 3), NAN), (1, (rows // 2, slice(None), 3), NAN), (2, (0, slice(None), 3), INF), (2, (1, slice(None), 3), NAN),
                           (2, (slice(None), slice(None), 3), INF), (2, (slice(0, None, 37), slice(None), 5), -INF), (0, (slice(None),), NAN), (2, (slice(None),), NAN)):
        x = [q, k, v]
        x[which] = x[which].clone()
        x[which][at] = bad
        spoilt = took(Call(*x, None, None).forward)
        assert spoilt < 5 * clean + 2, (which, bad, clean, spoilt)


def test_time_of_a_cache():
    for lengths, drafted in (([4000] * 16, [1] * 16), ([4000] * 4, [32] * 4)):
        c = Case(3, "bf16", lengths, drafted, 16, 4, 128, 64)
        clean = took(c.run)
        for which, bad in ((0, NAN), (1, INF), (1, NAN)):
            d = Case(3, "bf16", lengths, drafted, 16, 4, 128, 64)
            for s in range(len(lengths)):
                d.cache[which][int(d.table[s, 0]), :, 0, 3] = bad
            spoilt = took(d.run)
            assert not torch.isfinite(d.out).all()
            assert spoilt < 5 * clean + 2, (which, bad, clean, spoilt)
