"""Attention over packed prompts, forward and backward, against float64."""
import numpy as np
import pytest
import torch

from heads_helpers import B, DTYPES, assert_within, check_prompt, half_step, host, normal, oracle, qkv, starts

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


class Call:
    """A forward and a backward call with buffers that hold 7 and 0xFF before."""

    def __init__(self, q, k, v, q_starts, k_starts, causal=True, scale=None, grad=None):
        self.q, self.k, self.v, self.q_starts, self.k_starts, self.causal = q, k, v, q_starts, k_starts, causal
        self.scale = q.shape[2] ** -0.5 if scale is None else scale
        full = lambda t: torch.full(t.shape, 7.0, dtype=q.dtype, device="cuda")
        self.out, self.lse = full(q), torch.full((q.shape[1], q.shape[0]), 7.0, device="cuda")
        self.grad = grad
        if grad is not None:
            self.grads = [full(q), full(k), full(v)]
            self.ws = torch.full((B.dsq_attention_bwd_bytes(q.shape[0], q.shape[1]),), 0xFF, dtype=torch.uint8, device="cuda")

    def forward(self, stream=None):
        B.dsq_attention(self.q, self.k, self.v, self.q_starts, self.k_starts, self.causal, self.scale, self.out, self.lse, stream)
        return self

    def backward(self, stream=None):
        B.dsq_attention_bwd(self.q, self.k, self.v, self.out, self.lse, self.grad, self.q_starts, self.k_starts, self.causal, self.scale, *self.grads,
                            self.ws, stream)
        return self

    def check(self):
        at = lambda t, n: [0, n] if t is None else [min(max(i, 0), n) for i in t.tolist()]
        q_at = at(self.q_starts, len(self.q))
        k_at = at(self.k_starts if self.k_starts is not None else self.q_starts, len(self.k))
        check_prompt(self.q, self.k, self.v, q_at, k_at, self.causal, self.scale, self.out, self.lse, self.grad,
                     None if self.grad is None else self.grads, 7.0)


def call(seed, dtype, q_sizes, k_sizes, hq, hk, dim, causal=True, grad=True, first=0, behind=0, scale=None, spread=1.5):
    dt = DTYPES[dtype]
    rows, keys = first + sum(q_sizes) + behind, first + sum(k_sizes) + behind
    if q_sizes == k_sizes:
        q, k, v = qkv(seed, rows, hq, hk, dim, dt, spread)
    else:
        q, (k, v, _) = normal(seed, rows, hq, dim, dtype=dt, scale=spread), qkv(seed + 1, keys, hk, hk, dim, dt)
    single = len(q_sizes) == 1 and not first and not behind
    qs = None if single else starts(*q_sizes, first=first)
    ks = None if single or q_sizes == k_sizes else starts(*k_sizes, first=first)
    return Call(q, k, v, qs, ks, causal, scale, normal(seed + 2, rows, hq, dim, dtype=dt) if grad else None)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 300])
def test_lengths(n, causal, dtype):
    c = call(n, dtype, [n], [n], 2, 1, 64 if n % 2 else 128, causal)
    c.forward().backward().check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [8, 16, 24, 40, 64, 72, 80, 96, 112, 120, 128])
def test_dims(dim, dtype):
    c = call(dim, dtype, [70], [70], 3, 3, dim)
    c.forward().backward().check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hq,hk", [(1, 1), (8, 8), (8, 2), (7, 1), (12, 4), (16, 8), (24, 3), (9, 3)])
def test_heads(hq, hk, dtype):
    c = call(hq, dtype, [150], [150], hq, hk, 64)
    c.forward().backward().check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n,m", [(1, 300), (300, 1), (40, 170), (170, 40), (129, 128), (128, 129), (5, 260), (200, 64)])
def test_other_keys_than_rows(n, m, causal, dtype):
    """With more rows than keys the first rows of a causal call see nothing."""
    c = call(n + m, dtype, [n], [m], 4, 2, 64, causal)
    c.forward().backward().check()
    if causal and n > m:
        assert not c.out[:n - m].any() and torch.isneginf(c.lse[:, :n - m]).all() and not c.grads[0][:n - m].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("q_sizes,k_sizes", [((5, 0, 1, 130, 33), None), ((0, 0, 64), None), ((100, 3, 0), None), ((3, 40, 0, 129), (140, 40, 7, 0)), ((1,) * 70, None),
                                             ((0, 200, 1), (5, 100, 300))])
def test_packed(q_sizes, k_sizes, causal, dtype):
    """Empty sequences, sequences of one side, rows before the first and behind the last."""
    for first, behind in ((0, 0), (3, 11), (140, 1)):
        c = call(len(q_sizes) + first, dtype, list(q_sizes), list(k_sizes or q_sizes), 4, 2, 32, causal, first=first, behind=behind)
        c.forward().backward().check()


def test_more_sequences_than_a_wave_looks_at():
    """5000 sequences of one row: each is its own value."""
    c = call(1, "f32", [1] * 5000, [1] * 5000, 2, 1, 16)
    c.forward().backward()
    c.check()
    # p v / p: a product, a reciprocal and a product round
    want = host(c.v).repeat(2, axis=1)
    assert_within(host(c.out), want, 3.01 * oracle.U * np.abs(want), "values")


def test_one_long_sequence_among_many():
    sizes = [1] * 100 + [700] + [2] * 99
    c = call(2, "bf16", sizes, sizes, 2, 1, 64)
    c.forward().backward().check()


@pytest.mark.parametrize("dtype", DTYPES)
def test_long(dtype):
    """A few rows over many keys, and a causal prompt longer than a tile of the card: every eighth row by the oracle's float64."""
    c = call(4, dtype, [33], [5000], 2, 1, 128)
    c.forward().backward().check()
    c = call(5, dtype, [1500], [1500], 1, 1, 128)
    c.forward().backward().check()


@pytest.mark.parametrize("dtype", DTYPES)
def test_sharp_and_flat_scores(dtype):
    """Scores that rise along the keys, so that the running maximum is raised again and again; large ones; all the same."""
    dt = DTYPES[dtype]
    n = 200
    for kind in ("rising", "falling", "large", "same"):
        c = call(6, dtype, [n], [n], 2, 1, 64, causal=kind != "falling")
        c.q, c.k = c.q.contiguous(), c.k.contiguous()
        if kind in ("rising", "falling"):
            c.q[..., 0] = 8
            c.k[..., 0] = torch.linspace(-40, 40, n).to(dt)[:, None].cuda() * (1 if kind == "rising" else -1)
        elif kind == "large":
            c.q *= 8
            c.k *= 8
        else:
            c.k[:] = 0
        c.forward().backward().check()


@pytest.mark.parametrize("dtype", DTYPES)
def test_what_is_not_seen_has_no_part(dtype):
    """Infinities and NaN in keys and values of later tokens, of other sequences and behind the last: rows that do not see them are as without."""
    dt, sizes = DTYPES[dtype], [70, 50]
    for bad in (NAN, INF, -INF):
        c = call(7, dtype, sizes, sizes, 4, 2, 64, grad=False, behind=9)
        clean = Call(c.q, c.k, c.v, c.q_starts, None).forward()
        clean.check()
        c.k, c.v = c.k.contiguous(), c.v.contiguous()
        c.k[40, 0, 3] = c.v[45, 1, 5] = c.v[66, 0, 63] = bad
        c.k[120:], c.v[120:] = bad, bad
        c.forward()
        same = torch.ones(129, 4, dtype=torch.bool, device="cuda")
        same[40:70, :2] = same[45:70, 2:] = False
        # (a row beside a bad value is formed in another order: within the bounds, not to the bit)
        check_prompt(c.q, c.k.masked_fill(~torch.isfinite(c.k), 0), c.v.masked_fill(~torch.isfinite(c.v), 0), [0, 40], [0, 40], True, c.scale, c.out[:40], c.lse[:, :40])
        assert torch.equal(c.out[70:120], clean.out[70:120]) and (c.out[120:] == 7).all()
        assert torch.isfinite(c.out[:120][same[:120]]).all()
        half = half_step(dt)
        for h in (2, 3):
            r = oracle.attention(host(c.q)[:45, h], host(c.k)[:45, 1], host(c.v)[:45, 1], oracle.causal(45, 45), c.scale, half)
            assert_within(host(c.out)[:45, h], r["out"][0], r["out"][1] + half * np.abs(r["out"][0]) + half * r["out"][1] + 1e-7, "beside a bad value")
        assert not torch.isfinite(c.out[45:70, 2:, 5]).any()
        if bad is NAN:
            assert torch.isnan(c.out[40:70, :2]).all()


@pytest.mark.parametrize("dim", [72, 80, 96, 104, 128])
def test_binary32_keys_without_lds(dim):
    """Wide heads of few rows read keys and values straight from memory: odd lengths, blocks that end inside 32 keys, strides, a long row,
    and infinities and NaN behind what is seen."""
    for n, m, causal in ((1, 1, True), (3, 31, True), (33, 33, True), (63, 65, False), (31, 129, True), (129, 127, True), (100, 225, False)):
        c = call(n + m, "f32", [n], [m], 4, 2, dim, causal)
        c.forward().backward().check()
    c = call(1, "f32", [5, 0, 61, 1], [40, 3, 90, 1], 4, 2, dim, first=3, behind=2)
    c.forward().backward().check()
    # rows 2^24 elements and more apart: addresses of their own for each lane
    apart = torch.empty_strided((40, 2, dim), ((1 << 24) + 4, 128, 1), dtype=torch.float32, device="cuda")
    k = normal(2, 40, 2, dim, dtype=torch.float32)
    apart.copy_(k)
    q = normal(3, 40, 4, dim, dtype=torch.float32)
    a, b = Call(q, k, k, None, None).forward(), Call(q, apart, apart, None, None).forward()
    a.check()
    assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)
    for bad in (NAN, INF):
        c = call(4, "f32", [70], [70], 2, 1, dim, grad=False)
        clean = Call(c.q, c.k, c.v, None, None).forward()
        c.k, c.v = c.k.contiguous(), c.v.contiguous()
        c.k[50:], c.v[50:] = bad, bad
        c.forward()
        check_prompt(c.q, c.k[:50], c.v[:50], [0, 50], [0, 50], True, c.scale, c.out[:50], c.lse[:, :50])
        assert torch.equal(c.out[:32], clean.out[:32]) and not torch.isfinite(c.out[50:]).any()


def test_values_near_the_end_of_their_type():
    """Sums that pass the type's range on the way, not in the result."""
    for dt, big in ((torch.bfloat16, 3e38), (torch.float32, 3e38), (torch.float16, 6e4)):
        q, k, v = qkv(8, 100, 2, 1, 64, dt)
        v = torch.full_like(v, big).contiguous()
        c = Call(q, k, v, None, None).forward()
        assert torch.isfinite(c.out).all()
        assert ((c.out.double() / v.double() - 1).abs() < 4 * half_step(dt) + 200 * oracle.U).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides(dtype):
    dt, n, hq, hk, dim = DTYPES[dtype], 90, 4, 2, 48
    q, k, v = qkv(9, n, hq, hk, dim, dt)
    g = normal(10, n, hq, dim, dtype=dt)
    a = Call(*(t.contiguous() for t in (q, k, v)), None, None, grad=g).forward().backward()
    a.check()
    # heads before rows, for inputs and outputs, in wider rooms whose rest is left alone
    turned = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)
    b = Call(turned(q), turned(k), turned(v), None, None, grad=turned(g))
    rooms = [torch.full((t.shape[1], n, 64), 5.0, dtype=dt, device="cuda") for t in (q, q, k, v)]
    views = [r[:, :, 8:56].transpose(0, 1) for r in rooms]
    b.out, b.grads = views[0], views[1:]
    b.forward().backward()
    assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse) and all(torch.equal(x, y) for x, y in zip(a.grads, b.grads))
    assert all((r[..., :8] == 5).all() and (r[..., 56:] == 5).all() for r in rooms)
    # a key head that repeats for all, a query row that repeats
    wide = Call(q[:1].expand(n, -1, -1), k[:, :1].expand(-1, 2, -1), v[:, :1].expand(-1, 2, -1), None, None, grad=g[:, :1].expand(-1, hq, -1)).forward().backward()
    wide.check()


def test_far_apart():
    """Rows whose distance passes 2^32 bytes and 2^31 elements."""
    n, hq, dim = 70, 2, 32
    room = torch.zeros(70 * (1 << 25), dtype=torch.bfloat16, device="cuda")
    far = lambda at: room.as_strided((n, hq, dim), (1 << 25, dim, 1), at)
    q, k, v = qkv(11, n, hq, hq, dim, torch.bfloat16)
    g = normal(12, n, hq, dim, dtype=torch.bfloat16)
    near = Call(q, k, v, None, None, grad=g).forward().backward()
    c = Call(*(far(1024 * i) for i in range(3)), None, None, grad=far(4096))
    for t, x in ((c.q, q), (c.k, k), (c.v, v), (c.grad, g)):
        t.copy_(x)
    c.out, c.grads = far(8192), [far(8192 + 1024 * i) for i in range(1, 4)]
    c.forward().backward()
    assert torch.equal(c.out, near.out) and all(torch.equal(a, b) for a, b in zip(c.grads, near.grads))


def test_starts_outside_the_rows():
    """Starts past the rows are taken as their ends: nothing outside is read or written."""
    q, k, v = qkv(13, 50, 2, 1, 32, torch.float32)
    c = Call(q, k, v, torch.tensor([-5, 20, 90, 2 ** 31 - 1], dtype=torch.int32, device="cuda"), None, grad=normal(14, 50, 2, 32)).forward().backward()
    c.check()
    d = Call(q, k, v, torch.tensor([30, 10, 40, 20], dtype=torch.int32, device="cuda"), None, grad=c.grad).forward().backward()
    torch.cuda.synchronize()
    assert (d.out[45:] == 7).all()


def test_same_bits_every_time():
    for dtype in DTYPES:
        c = call(15, dtype, [300, 40], [300, 40], 8, 2, 64)
        c.forward().backward()
        first = [t.clone() for t in [c.out, c.lse] + c.grads]
        for _ in range(3):
            c.ws.fill_(0xFF)
            c.forward().backward()
            assert all(torch.equal(a, b) for a, b in zip(first, [c.out, c.lse] + c.grads))


def test_without_lse():
    c = call(16, "bf16", [100], [100], 4, 2, 64, grad=False)
    c.forward()
    out = torch.empty_like(c.out)
    B.dsq_attention(c.q, c.k, c.v, None, None, True, c.scale, out, None)
    assert torch.equal(out, c.out)


def test_gradients_against_differences():
    """Gradients against central differences of the float64 oracle: binary32 arithmetic leaves some 1e-5 of sums of hundreds of terms."""
    c = call(17, "f32", [25, 18], [30, 12], 4, 2, 24)
    c.forward().backward()
    x = [host(t) for t in (c.q, c.k, c.v)]
    g = host(c.grad)

    def loss(q, k, v):
        total = 0.0
        for (a, b), (s, e) in (((0, 25), (0, 30)), ((25, 43), (30, 42))):
            for h in range(4):
                total += (g[a:b, h] * oracle.attention(q[a:b, h], k[s:e, h // 2], v[s:e, h // 2], oracle.causal(b - a, e - s), c.scale, 0.0)["out"][0]).sum()
        return total

    rs = np.random.RandomState(2)
    for at, got in enumerate(c.grads):
        for _ in range(3):
            d = rs.randn(*got.shape)
            up, down = list(x), list(x)
            up[at], down[at] = x[at] + 1e-6 * d, x[at] - 1e-6 * d
            diff = (loss(*up) - loss(*down)) / 2e-6
            assert abs(diff - (host(got) * d).sum()) <= 1e-5 * np.abs(host(got) * d).sum()


def test_nothing_to_do():
    e = torch.empty(0, 2, 32, device="cuda")
    k = torch.full((5, 1, 32), 2.0, device="cuda")
    B.dsq_attention(e, k, k, None, None, True, 1.0, e, None)
    # rows without keys are zeros, keys without rows have gradients of zero
    q = torch.ones(5, 2, 32, device="cuda")
    none = torch.empty(0, 1, 32, device="cuda")
    c = Call(q, none, none, None, None, grad=q).forward().backward()
    assert not c.out.any() and torch.isneginf(c.lse).all() and not c.grads[0].any()
    c = Call(e, k, k, None, None, grad=e)
    c.ws = None
    c.backward()
    assert not c.grads[1].any() and not c.grads[2].any()
    # no sequences
    c = call(18, "f32", [], [], 2, 1, 32, behind=4)
    c.forward().backward()
    assert (c.out == 7).all() and all((t == 7).all() for t in c.grads)
