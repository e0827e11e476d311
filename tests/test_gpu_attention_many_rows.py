"""Attention over prompts of many rows: the kernels that own 128 rows a workgroup (64 in the binary32 backward pass), against float64.
test_attn_prompt_plan.py holds that these shapes take those kernels."""
import numpy as np
import pytest
import torch

from heads_helpers import B, DTYPES, check_prompt, host, normal, oracle, qkv, starts
from test_gpu_attention import Call, call

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")

# name: rows of the sequences, keys of the sequences (None: as the rows), query heads, key heads, rows before the first sequence
SHAPES = {
    "one": ([1030], None, 48, 6, 0),
    "packed": ([0, 1, 257, 130, 0, 64, 129, 500, 33, 0], None, 48, 12, 0),
    "other keys": ([300, 1, 0, 200, 127, 396], [40, 500, 30, 200, 300, 0], 48, 16, 0),
    "behind others": ([128, 256, 640], None, 50, 5, 37),
    "short": ([5] * 140 + [64] * 3, None, 60, 4, 3),
}
DIMS = [40, 64, 80, 96, 104, 128]


def check_heads(c, pairs):
    """Key heads `pairs` with the query heads that share them."""
    group = c.q.shape[1] // c.k.shape[1]
    at = lambda t, n: [0, n] if t is None else t.tolist()
    q_at = at(c.q_starts, len(c.q))
    k_at = at(c.k_starts, len(c.k)) if c.k_starts is not None else q_at if c.q_starts is not None else [0, len(c.k)]
    for kv in pairs:
        h, k = slice(kv * group, (kv + 1) * group), slice(kv, kv + 1)
        grads = None if c.grad is None else [c.grads[0][:, h], c.grads[1][:, k], c.grads[2][:, k]]
        check_prompt(c.q[:, h], c.k[:, k], c.v[:, k], q_at, k_at, c.causal, c.scale, c.out[:, h], c.lse[h], None if c.grad is None else c.grad[:, h], grads, 7.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("name", SHAPES)
def test_shapes(name, dim, dtype):
    q_sizes, k_sizes, hq, hk, first = SHAPES[name]
    c = call(dim, dtype, q_sizes, k_sizes or q_sizes, hq, hk, dim, name != "behind others", first=first, behind=first)
    c.forward().backward()
    check_heads(c, range(hk) if dim == 64 else (0, hk - 1))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_not_causal(dim, dtype):
    """Keys that fill their last tile and that do not."""
    for n, m in ((1024, 128), (1100, 65), (1100, 1), (1024, 300)):
        c = call(dim + m, dtype, [n], [m], 48, 3, dim, False)
        c.forward().backward()
        check_heads(c, (0, 2))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [64, 80, 128])
def test_both_sides_of_the_limit(dim, dtype):
    """As many rows times heads as the last call of the one kind and the first of the other have: the same results within the bounds."""
    for rows, heads in ((682, 48), (683, 48), (1023, 48), (1024, 48)):
        c = call(dim, dtype, [rows], [rows], heads, 6, dim)
        c.forward().backward()
        check_heads(c, (5,))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [64, 80, 128])
def test_sharp_scores(dim, dtype):
    """Scores that rise and fall along the keys: the running maximum is raised again and again."""
    dt, n = DTYPES[dtype], 1100
    for up in (1, -1):
        c = call(3, dtype, [n], [n], 48, 4, dim, up > 0)
        c.q, c.k = c.q.contiguous(), c.k.contiguous()
        c.q[..., 0] = 8
        c.k[..., 0] = torch.linspace(-40, 40, n).to(dt)[:, None].cuda() * up
        c.forward().backward()
        check_heads(c, (0, 3))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [64, 80, 96, 128])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_what_is_not_seen_has_no_part(bad, dim, dtype):
    """Bad keys and values in the middle of a prompt, of another sequence and behind the last: rows that do not see them are as without."""
    sizes = [600, 380]
    c = call(4, dtype, sizes, sizes, 48, 4, dim, grad=False, behind=70)
    clean = Call(c.q, c.k, c.v, c.q_starts, None).forward()
    c.k, c.v = c.k.contiguous(), c.v.contiguous()
    c.k[333, 0, 3] = c.v[340, 1, 5] = c.v[345, 3, dim - 1] = bad
    c.k[980:], c.v[980:] = bad, bad
    c.forward()
    assert torch.equal(c.out[600:980], clean.out[600:980]) and (c.out[980:] == 7).all()
    assert torch.equal(c.out[:, 24:36], clean.out[:, 24:36])
    for kv, last in ((0, 333), (1, 340), (3, 345)):
        h, k = slice(12 * kv, 12 * kv + 12), slice(kv, kv + 1)
        check_prompt(c.q[:last, h], c.k[:last, k], c.v[:last, k], [0, last], [0, last], True, c.scale, c.out[:last, h], c.lse[h, :last])
    assert not torch.isfinite(c.out[340:600, 12:24, 5]).any() and not torch.isfinite(c.out[345:600, 36:, dim - 1]).any()
    if bad is NAN:
        assert torch.isnan(c.out[333:600, :12]).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_and_repeats(dtype):
    """Heads before rows in wider rooms, keys far apart (addresses of each lane's own), a key head that repeats."""
    dt, n, hq, hk, dim = DTYPES[dtype], 1100, 48, 4, 64
    q, k, v = qkv(5, n, hq, hk, dim, dt)
    g = normal(6, n, hq, dim, dtype=dt)
    a = Call(*(t.contiguous() for t in (q, k, v)), None, None, grad=g).forward().backward()
    check_heads(a, (0, 3))
    turned = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)
    b = Call(turned(q), turned(k), turned(v), None, None, grad=turned(g))
    rooms = [torch.full((t.shape[1], n, 80), 5.0, dtype=dt, device="cuda") for t in (q, q, k, v)]
    views = [r[:, :, 8:72].transpose(0, 1) for r in rooms]
    b.out, b.grads = views[0], views[1:]
    b.forward().backward()
    assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse) and all(torch.equal(x, y) for x, y in zip(a.grads, b.grads))
    assert all((r[..., :8] == 5).all() and (r[..., 72:] == 5).all() for r in rooms)
    # 140 keys 2^24 elements and more apart
    apart = torch.empty_strided((140, hk, dim), ((1 << 24) + 8, dim, 1), dtype=dt, device="cuda")
    apart.copy_(k[:140])
    near = Call(q, k[:140].contiguous(), k[:140].contiguous(), None, None, causal=False, grad=g).forward().backward()
    check_heads(near, (1,))
    far = Call(q, apart, apart, None, None, causal=False, grad=g).forward()
    assert torch.equal(near.out, far.out) and torch.equal(near.lse, far.lse)
    far.grads[1:] = [torch.full((140, hk, dim), 7.0, dtype=dt, device="cuda") for _ in "kv"]
    far.backward()
    assert all(torch.equal(x, y) for x, y in zip(near.grads, far.grads))
    one = Call(q, k[:, :1].expand(-1, hk, -1), v[:, :1].expand(-1, hk, -1), None, None, grad=g).forward().backward()
    check_heads(one, (0, 2))


def test_same_bits_every_time():
    for dtype in DTYPES:
        c = call(15, dtype, [900, 140], [900, 140], 48, 4, 64)
        c.forward().backward()
        first = [t.clone() for t in [c.out, c.lse] + c.grads]
        for _ in range(3):
            c.ws.fill_(0xFF)
            c.forward().backward()
            assert all(torch.equal(a, b) for a, b in zip(first, [c.out, c.lse] + c.grads))


def test_gradients_against_differences():
    """Directional derivatives of the float64 formula: binary32 arithmetic leaves some 1e-5 of sums of thousands of terms."""
    c = call(17, "f32", [600, 430], [600, 430], 48, 3, 64)
    c.forward().backward()
    x, g = [host(t) for t in (c.q, c.k, c.v)], host(c.grad)
    heads = (0, 20, 47)

    def loss(q, k, v):
        total = 0.0
        for s, e in ((0, 600), (600, 1030)):
            for h in heads:
                total += (g[s:e, h] * oracle.attention(q[s:e, h], k[s:e, h // 16], v[s:e, h // 16], oracle.causal(e - s, e - s), c.scale, 0.0)["out"][0]).sum()
        return total

    # the loss of three heads alone: the gradient of the call with the other heads' gradients zero
    c.grad = c.grad.clone()
    c.grad[:, [h for h in range(48) if h not in heads]] = 0
    c.backward()
    rs = np.random.RandomState(2)
    for at, got in enumerate(c.grads):
        d = rs.randn(*got.shape)
        up, down = list(x), list(x)
        up[at], down[at] = x[at] + 1e-6 * d, x[at] - 1e-6 * d
        diff = (loss(*up) - loss(*down)) / 2e-6
        assert abs(diff - (host(got) * d).sum()) <= 1e-5 * np.abs(host(got) * d).sum()
