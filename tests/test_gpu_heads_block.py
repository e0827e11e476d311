"""The calls for heads as they are used: with the norm and the 4-bit products in a serving step and in a training step, in graphs, on
streams, both ways of the binding, and refused."""
import numpy as np
import pytest
import torch

from heads_helpers import B, DTYPES, assert_within, check_prompt, check_rope, half_step, host, normal, operand_tiny, oracle, rotation, starts, tiny
from lm_helpers import pack, random_w4
from test_gpu_head_rope import check_grads
from test_gpu_lm_layers import General

pytestmark = pytest.mark.gpu
EPS = 1e-6
WIDTH, HQ, HK, DIM, PAGE = 256, 4, 2, 64, 16


class Block:
    """A block's attention: norm, q/k/v product, norms of heads with rotation, cache, attention, output product; a prompt of each
    sequence first, then drafted tokens.  ``tokens``: of each sequence and step."""

    def __init__(self, dtype, prompt, drafted, seed=1, tree=True):
        dt = self.dt = DTYPES[dtype]
        e = lambda *s, **k: torch.empty(*s, device="cuda", **{"dtype": dt, **k})
        self.group = 64
        self.w_qkv = pack(*random_w4(seed, (HQ + 2 * HK) * DIM, WIDTH, self.group), self.group)
        self.w_out = pack(*random_w4(seed + 1, WIDTH, HQ * DIM, self.group), self.group)
        self.wn, self.qw, self.kw = (normal(seed + i, n, dtype=dt) for i, n in ((2, WIDTH), (3, DIM), (4, DIM)))
        self.sizes = [prompt, drafted]
        total = [a + b for a, b in zip(prompt, drafted)]
        need = [-(-n // PAGE) for n in total]
        order = np.random.RandomState(seed).permutation(sum(need) + 2)[:sum(need)]
        self.table = torch.full((len(total), max(need)), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = torch.tensor(order[at:at + n].astype(np.int32))
            at += n
        self.cache = [torch.full((sum(need) + 2, HK, PAGE, DIM), float("nan"), dtype=dt, device="cuda") for _ in "kv"]
        self.steps = []
        for step, (sizes, before) in enumerate(((prompt, [0] * len(prompt)), (drafted, prompt))):
            rows = sum(sizes)
            place = np.concatenate([np.arange(n) + b for n, b in zip(sizes, before)])
            of = np.repeat(np.arange(len(sizes)), sizes)
            slots = self.table[of, place // PAGE].long() * PAGE + torch.tensor(place % PAGE)
            turning = rotation(2, rows, DIM)
            turning = (torch.tensor(place[None].astype(np.int32), device="cuda"),) + turning[1:]
            self.steps.append(dict(x=normal(seed + 5 + step, rows, WIDTH, dtype=dt), y=e(rows, WIDTH), qkv=e(rows, (HQ + 2 * HK) * DIM), q=e(rows, HQ, DIM),
                                   k=e(rows, HK, DIM), slots=slots.cuda(), turning=turning, a=e(rows, HQ, DIM), out=e(rows, WIDTH), starts=starts(*sizes)))
        self.table = self.table.cuda()
        self.lengths = torch.tensor(total, dtype=torch.int32, device="cuda")
        self.tree = None
        if tree:
            rs = np.random.RandomState(seed)
            self.words = [np.array([[1 << i | int(rs.randint(0, 1 << 62)) & (1 << i) - 1] for i in range(n)], np.uint64).reshape(n, 1) for n in drafted]
            self.tree = torch.tensor(np.concatenate(self.words).view(np.int64), device="cuda")
        self.most = max(drafted)
        self.ws = e(B.dsq_attention_cache_bytes(len(total), self.most, HQ, HK, DIM), dtype=torch.uint8)
        self.scale = DIM ** -0.5

    def step(self, i, stream=None):
        s = self.steps[i]
        B.dsq_rms_norm(s["x"], None, self.wn, EPS, None, s["y"], None, None, None, stream)
        B.dsq_linear_w4(s["y"], *self.w_qkv, (HQ + 2 * HK) * DIM, WIDTH, self.group, None, s["qkv"], stream)
        heads = s["qkv"].view(-1, HQ + 2 * HK, DIM)
        q, k, v = heads[:, :HQ], heads[:, HQ:HQ + HK], heads[:, HQ + HK:]
        B.dsq_qk_norm_rope(q, k, v, self.qw, self.kw, EPS, *s["turning"], False, s["q"], s["k"] if i == 0 else None, *self.cache, s["slots"], stream)
        if i == 0:
            B.dsq_attention(s["q"], s["k"], v, s["starts"], None, True, self.scale, s["a"], None, stream)
        else:
            B.dsq_attention_cache(s["q"], s["starts"], self.most, *self.cache, self.table, self.lengths, self.tree, self.scale, s["a"], self.ws, stream)
        B.dsq_linear_w4(s["a"].view(-1, HQ * DIM), *self.w_out, WIDTH, HQ * DIM, self.group, None, s["out"], stream)

    def run(self, stream=None):
        self.step(0, stream)
        self.step(1, stream)
        return self

    def outputs(self):
        return [s[n] for s in self.steps for n in ("y", "qkv", "q", "a", "out")] + [self.steps[0]["k"]]

    def results(self):
        torch.cuda.synchronize()
        return [t.clone() for t in self.outputs()] + [t.nan_to_num().clone() for t in self.cache]

    def scramble(self):
        for t in self.outputs() + self.cache:
            t.fill_(float("nan"))
        self.ws.fill_(0xFF)

    def check(self):
        torch.cuda.synchronize()
        for i, s in enumerate(self.steps):
            heads = s["qkv"].view(-1, HQ + 2 * HK, DIM)
            check_rope(heads[:, :HQ], self.qw, EPS, s["turning"], False, s["q"], "q")
            rows = [c.transpose(1, 2).reshape(-1, HK, DIM)[s["slots"]] for c in self.cache]
            check_rope(heads[:, HQ:HQ + HK], self.kw, EPS, s["turning"], False, rows[0], "cached k")
            assert torch.equal(rows[1], heads[:, HQ + HK:])
        s = self.steps[0]
        check_prompt(s["q"], s["k"], s["qkv"].view(-1, HQ + 2 * HK, DIM)[:, HQ + HK:], s["starts"].tolist(), s["starts"].tolist(), True, self.scale, s["a"])
        s, at, half = self.steps[1], 0, half_step(self.dt)
        q, a = host(s["q"]), host(s["a"])
        for i, (p, n) in enumerate(zip(*self.sizes)):
            page = self.table[i, :-(-(p + n) // PAGE)].long()
            k, v = (host(c[page].transpose(1, 2).reshape(-1, HK, DIM)[:p + n]) for c in self.cache)
            seen = oracle.tree_mask(n, p + n, None if self.tree is None else self.words[i])
            for h in range(HQ):
                want, bound = oracle.attention(q[at:at + n, h], k[:, h // 2], v[:, h // 2], seen, self.scale, half, tiny=operand_tiny(self.dt))["out"]
                assert_within(a[at:at + n, h], want, bound + half * (np.abs(want) + bound) + tiny(self.dt), "drafted")
            at += n


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tree", [True, False])
def test_serving(tree, dtype):
    for prompt, drafted in (([5], [1]), ([40, 1, 130], [3, 8, 1]), ([300, 17], [1, 1])):
        Block(dtype, prompt, drafted, tree=tree).run().check()


@pytest.mark.parametrize("dtype", DTYPES)
def test_the_cache_and_the_prompt_agree(dtype):
    """A chain of drafted tokens sees what the end of a causal prompt sees."""
    b = Block(dtype, [100], [20], tree=False).run()
    k, v = (c[b.table[0].long()].transpose(1, 2).reshape(-1, HK, DIM)[:120].contiguous() for c in b.cache)
    out = torch.empty_like(b.steps[1]["a"])
    B.dsq_attention(b.steps[1]["q"], k, v, None, None, True, b.scale, out, None)
    far = (out.double() - b.steps[1]["a"].double()).abs()
    assert (far <= 4 * half_step(b.dt) * (out.double().abs() + v.double().abs().max()) + 1e-5).all()


def test_serving_in_graphs_and_on_other_streams():
    a, b = Block("bf16", [40, 130], [3, 8]), Block("f16", [70, 2000, 1], [2, 1, 4], seed=50)
    want_a, want_b = a.run().results(), b.run().results()
    same = lambda: all(torch.equal(x, y) for x, y in zip(a.results() + b.results(), want_a + want_b))
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for t in (s1, s2.cuda_stream):
        a.scramble()
        torch.cuda.synchronize()
        a.run(t)
        assert same()
    a.scramble(), b.scramble()
    torch.cuda.synchronize()
    for _ in range(3):
        for one, s in ((a, s1), (b, s2)):
            with torch.cuda.stream(s):
                one.run()
    assert same()
    graphs = []
    for one, s in ((a, s1), (b, s2)):
        with torch.cuda.stream(s):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                one.run()
            graphs.append(g)
    for i in range(3):
        a.scramble(), b.scramble()
        torch.cuda.synchronize()
        graphs[i % 2].replay()
        graphs[1 - i % 2].replay()
        assert same()
        a.run()                                             # eager work between the replays
        assert same()
    # other lengths and inputs in the same places
    a.steps[0]["x"].copy_(normal(77, 170, WIDTH, dtype=a.dt))
    graphs[0].replay()
    a.check()


class Training:
    """Heads through norm and rotation, attention and back."""

    def __init__(self, dtype, sizes, seed=1):
        dt, rows = DTYPES[dtype], sum(sizes)
        e = lambda *s, **k: torch.empty(*s, device="cuda", **{"dtype": dt, **k})
        self.qkv = normal(seed, rows, HQ + 2 * HK, DIM, dtype=dt)
        self.qw, self.kw = normal(seed + 1, DIM, dtype=dt), normal(seed + 2, DIM, dtype=dt)
        self.turning, self.starts, self.scale = rotation(3, rows, 48, 2), starts(*sizes), DIM ** -0.5
        self.grad = normal(seed + 3, rows, HQ, DIM, dtype=dt)
        self.q, self.k, self.a, self.gq, self.gk = e(rows, HQ, DIM), e(rows, HK, DIM), e(rows, HQ, DIM), e(rows, HQ, DIM), e(rows, HK, DIM)
        self.lse, self.gqw, self.gkw = e(HQ, rows, dtype=torch.float32), e(DIM, dtype=torch.float32), e(DIM, dtype=torch.float32)
        self.gqkv = e(rows, HQ + 2 * HK, DIM)
        n = max(B.dsq_attention_bwd_bytes(rows, HQ), B.dsq_qk_norm_rope_bwd_bytes(rows, HQ, HK, DIM))
        self.ws = e(n, dtype=torch.uint8)                    # of calls that follow one another

    def parts(self, t):
        return t[:, :HQ], t[:, HQ:HQ + HK], t[:, HQ + HK:]

    def run(self):
        (q, k, v), (gq, gk, gv) = self.parts(self.qkv), self.parts(self.gqkv)
        B.dsq_qk_norm_rope(q, k, None, self.qw, self.kw, EPS, *self.turning, True, self.q, self.k, None, None, None)
        B.dsq_attention(self.q, self.k, v, self.starts, None, True, self.scale, self.a, self.lse)
        B.dsq_attention_bwd(self.q, self.k, v, self.a, self.lse, self.grad, self.starts, None, True, self.scale, self.gq, self.gk, gv, self.ws)
        B.dsq_qk_norm_rope_bwd(q, k, self.qw, self.kw, EPS, *self.turning, True, self.gq, self.gk, gq, gk, self.gqw, self.gkw, self.ws)
        return self

    def outputs(self):
        return [self.q, self.k, self.a, self.gq, self.gk, self.lse, self.gqw, self.gkw, self.gqkv]

    def results(self):
        torch.cuda.synchronize()
        return [t.clone() for t in self.outputs()]

    def scramble(self):
        for t in self.outputs():
            t.fill_(float("nan"))
        self.ws.fill_(0xFF)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("sizes", [(1,), (50, 130), (300, 1, 20)])
def test_training(sizes, dtype):
    t = Training(dtype, list(sizes)).run()
    q, k, v = t.parts(t.qkv)
    check_rope(q, t.qw, EPS, t.turning, True, t.q, "q")
    check_rope(k, t.kw, EPS, t.turning, True, t.k, "k")
    gq, gk, gv = t.parts(t.gqkv)
    at = t.starts.tolist()
    check_prompt(t.q, t.k, v, at, at, True, t.scale, t.a, t.lse, t.grad, [t.gq, t.gk, gv])
    check_grads(q, t.qw, EPS, t.turning, True, t.gq, gq, t.gqw, 512, "q")
    check_grads(k, t.kw, EPS, t.turning, True, t.gk, gk, t.gkw, 512, "k")


def test_training_against_differences():
    """The whole chain against central differences of the float64 oracle: binary32 arithmetic leaves some 1e-5."""
    t = Training("f32", [13, 20]).run()
    torch.cuda.synchronize()
    angle = oracle.angles(host(t.turning[0]).astype(np.int64), t.turning[1].cpu().numpy(), host(t.turning[2]))
    g = host(t.grad)

    def loss(x, qw, kw):
        q, k = oracle.norm_rope(x[:, :HQ], qw, EPS, angle, True)[0], oracle.norm_rope(x[:, HQ:HQ + HK], kw, EPS, angle, True)[0]
        return sum((g[a:b, h] * oracle.attention(q[a:b, h], k[a:b, h // 2], x[a:b, HQ + HK + h // 2], oracle.causal(b - a, b - a), t.scale, 0.0)["out"][0]).sum()
                   for a, b in ((0, 13), (13, 33)) for h in range(HQ))

    rs = np.random.RandomState(3)
    for at, got in enumerate((t.gqkv, t.gqw, t.gkw)):
        for _ in range(4):
            d = rs.randn(*got.shape)
            up, down = [host(t.qkv), host(t.qw), host(t.kw)], [host(t.qkv), host(t.qw), host(t.kw)]
            up[at], down[at] = up[at] + 1e-6 * d, down[at] - 1e-6 * d
            diff = (loss(*up) - loss(*down)) / 2e-6
            assert abs(diff - (host(got) * d).sum()) <= 2e-5 * np.abs(host(got) * d).sum()


def test_training_in_graphs():
    """Two captured steps with a workspace each, replayed at once, and an eager one between."""
    a, b = Training("bf16", [150, 200]), Training("f32", [33, 300], seed=50)
    want_a, want_b = a.run().results(), b.run().results()
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for one, s in zip((a, b), streams):
        with torch.cuda.stream(s):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                one.run()
            graphs.append(g)
    for _ in range(3):
        a.scramble(), b.scramble()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        assert all(torch.equal(x, y) for x, y in zip(a.results() + b.results(), want_a + want_b))
        assert all(torch.equal(x, y) for x, y in zip(b.run().results(), want_b))


def test_no_rows_in_a_graph():
    e, gw = torch.empty(0, 2, 32, device="cuda"), torch.full((32,), 3.0, device="cuda")
    turning = rotation(2, 0, 32)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            B.dsq_qk_norm_rope_bwd(e, e, None, None, EPS, *turning, False, e, e, e, e, gw, None, None)
        for _ in range(3):
            gw.fill_(5.0)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert not gw.any()


def test_both_ways_of_the_binding(monkeypatch):
    runs = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(B, "_marshal", General())
        b, t = Block("f16", [20, 70], [3, 1]).run(), Training("f32", [40, 9]).run()
        p = Block("bf16", [20, 70], [1, 1], tree=False)
        p.run(torch.cuda.current_stream())
        one, other = torch.empty_like(t.q), torch.empty_like(t.k)
        B.dsq_qk_norm_rope(t.q, None, None, None, None, 0.0, t.turning[0][0].contiguous(), None, t.turning[2], 1, one, None, None, None, None)
        B.dsq_qk_norm_rope(None, t.k, None, None, None, 0, None, None, None, 0, None, other, None, None, None)
        assert torch.equal(other, t.k)
        runs.append(b.results() + t.results() + p.results() + [one.clone()])
    assert all(torch.equal(x, y) for x, y in zip(*runs))


@pytest.mark.parametrize("native", [True, False])
def test_refused_calls_write_nothing(native, monkeypatch):
    if not native:
        monkeypatch.setattr(B, "_marshal", General())
    b, t = Block("bf16", [20, 70], [3, 1]).run(), Training("bf16", [40, 9]).run()
    torch.cuda.synchronize()
    outs = b.outputs() + b.cache + t.outputs() + [b.ws, t.ws]
    for i, o in enumerate(outs):
        o.fill_(i + 3)
    before = [o.clone() for o in outs]
    s = b.steps[1]
    heads = s["qkv"].view(-1, HQ + 2 * HK, DIM)
    f = lambda v: v.float()
    rope = lambda q=heads[:, :HQ], k=heads[:, HQ:HQ + HK], v=heads[:, HQ + HK:], qw=b.qw, kw=b.kw, eps=EPS, p=s["turning"][0], pa=None, fr=s["turning"][2], il=False, \
        qo=s["q"], ko=None, kc=b.cache[0], vc=b.cache[1], sl=s["slots"]: B.dsq_qk_norm_rope(q, k, v, qw, kw, eps, p, pa, fr, il, qo, ko, kc, vc, sl)
    cache = lambda q=s["q"], st=s["starts"], most=3, kc=b.cache[0], vc=b.cache[1], tb=b.table, n=b.lengths, tr=b.tree, sc=0.1, o=s["a"], ws=b.ws: \
        B.dsq_attention_cache(q, st, most, kc, vc, tb, n, tr, sc, o, ws)
    v = t.parts(t.qkv)[2]
    gq, gk, gv = t.parts(t.gqkv)
    attn = lambda q=t.q, k=t.k, v=v, qs=t.starts, ks=None, ca=True, sc=0.1, o=t.a, l=t.lse: B.dsq_attention(q, k, v, qs, ks, ca, sc, o, l)
    attn_bwd = lambda q=t.q, k=t.k, v=v, o=t.a, l=t.lse, g=t.grad, qs=t.starts, ks=None, sc=0.1, gq=t.gq, gk=t.gk, gv=gv, ws=t.ws: \
        B.dsq_attention_bwd(q, k, v, o, l, g, qs, ks, True, sc, gq, gk, gv, ws)
    rope_bwd = lambda q=t.qkv[:, :HQ], k=t.qkv[:, HQ:HQ + HK], qw=t.qw, kw=t.kw, eps=EPS, p=t.turning[0], pa=t.turning[1], fr=t.turning[2], go=t.gq, gko=t.gk, gq=gq, gk=gk, \
        gqw=t.gqw, gkw=t.gkw, ws=t.ws: B.dsq_qk_norm_rope_bwd(q, k, qw, kw, eps, p, pa, fr, True, go, gko, gq, gk, gqw, gkw, ws)
    odd = torch.empty(4 * HQ * DIM + 8, dtype=b.dt, device="cuda")[1:1 + 4 * HQ * DIM].view(4, HQ, DIM)
    stat = lambda *calls: [(c, n) for n, group in calls for c in group]
    for call, status in stat(
            (1, [lambda: rope(q=None, qo=s["q"], k=None), lambda: rope(sl=None), lambda: rope(vc=None), lambda: rope(kc=None), lambda: rope(v=None), lambda: rope(fr=s["turning"][2], p=None),
                 lambda: attn(q=None), lambda: attn(k=None), lambda: attn(o=None), lambda: attn(qs=None, ks=t.starts[:2]), lambda: attn_bwd(l=None), lambda: attn_bwd(ws=None), lambda: attn_bwd(gk=None),
                 lambda: rope_bwd(gq=None), lambda: rope_bwd(ws=None), lambda: cache(q=None), lambda: cache(n=None), lambda: cache(ws=None), lambda: cache(tb=None), lambda: cache(kc=None)]),
            (3, [lambda: rope(eps=-1.0), lambda: attn(sc=0.0), lambda: attn(sc=float("nan")), lambda: attn_bwd(sc=-0.1), lambda: cache(sc=float("inf")), lambda: rope_bwd(eps=float("inf"))]),
            (4, [lambda: rope(k=heads[:2, HQ:HQ + HK]), lambda: rope(k=heads[:, HQ:HQ + HK, :32]), lambda: rope(qw=b.qw[:8]), lambda: rope(p=s["turning"][0][:, :3]),
                 lambda: rope(qo=s["q"][:3]), lambda: rope(sl=s["slots"][:2]), lambda: rope(kc=b.cache[0][:, :1].contiguous()), lambda: rope(vc=b.cache[1][:3]),
                 lambda: rope(qo=s["q"][:, :1].expand(-1, HQ, -1)), lambda: rope(fr=torch.ones(40, device="cuda"), pa=None), lambda: rope(pa=torch.zeros(31, dtype=torch.uint8, device="cuda")),
                 lambda: attn(k=t.k[..., :32]), lambda: attn(v=v[:-1]), lambda: attn(o=t.a[:-1]), lambda: attn(l=t.lse[:-1]), lambda: attn(ks=t.starts[:2]), lambda: attn(q=t.q[0]),
                 lambda: attn(q=t.q[:, :3], o=t.a[:, :3], l=None), lambda: attn_bwd(g=t.grad[1:]), lambda: attn_bwd(gv=gv[:, :1]), lambda: attn_bwd(gk=t.gk[:1].expand(49, -1, -1)),
                 lambda: rope_bwd(go=t.gq[1:]), lambda: rope_bwd(gqw=t.gqw[:8]), lambda: cache(tr=b.tree[:2]), lambda: cache(tr=b.tree[:, :0]), lambda: cache(st=s["starts"][:2]),
                 lambda: cache(tb=b.table[:1]), lambda: cache(kc=b.cache[0][:, :, :, :32].contiguous()), lambda: cache(vc=b.cache[1][:2]), lambda: cache(most=0), lambda: cache(st=None), lambda: cache(o=s["a"][:1])]),
            (5, [lambda: rope(eps=0.0), lambda: rope(fr=torch.ones(20, device="cuda")), lambda: rope_bwd(eps=0.0), lambda: rope(kc=torch.zeros(4, HK, 24, DIM, dtype=b.dt, device="cuda"), vc=torch.zeros(4, HK, 24, DIM, dtype=b.dt, device="cuda"))]),
            (6, [lambda: rope(q=odd), lambda: cache(q=odd), lambda: attn(q=odd, o=t.a[:4], l=None)]),
            (7, [lambda: attn_bwd(ws=t.ws[:64]), lambda: rope_bwd(ws=t.ws[:64]), lambda: cache(ws=b.ws[:64])])):
        with pytest.raises(B.DsqError) as e:
            call()
        assert e.value.status == status, (status, str(e.value))
    for call in (lambda: rope(q=f(heads[:, :HQ])), lambda: rope(v=f(heads[:, HQ + HK:])), lambda: rope(qw=f(b.qw)), lambda: rope(p=s["turning"][0].long()), lambda: rope(sl=s["slots"].int()),
                 lambda: rope(kc=f(b.cache[0])), lambda: rope(q=heads[:, :HQ].cpu()), lambda: rope(qo=s["q"].transpose(1, 2).contiguous().transpose(1, 2)), lambda: rope(fr=s["turning"][2].double()),
                 lambda: attn(k=f(t.k)), lambda: attn(q=t.q.double()), lambda: attn(l=t.lse.half()), lambda: attn(qs=t.starts.long()), lambda: attn_bwd(g=f(t.grad)), lambda: attn_bwd(gv=f(gv)),
                 lambda: rope_bwd(gqw=t.gqw.half()), lambda: rope_bwd(ws=t.ws.view(torch.int8)), lambda: cache(tb=b.table.long()), lambda: cache(n=b.lengths.long()), lambda: cache(tr=b.tree.int()),
                 lambda: cache(kc=b.cache[0].transpose(1, 2).contiguous().transpose(1, 2)), lambda: cache(o=f(s["a"])), lambda: cache(tb=b.table.t().contiguous().t())):
        with pytest.raises(TypeError):
            call()
    torch.cuda.synchronize()
    for i, (o, want) in enumerate(zip(outs, before)):
        assert torch.equal(o, want), i
    # (the same calls with their own arguments do write)
    rope(), cache(), attn(), attn_bwd(), rope_bwd()
    torch.cuda.synchronize()
    for o in (s["q"], s["a"], t.a, t.gq, t.gqkv, t.gqw, b.cache[0]):
        i = [x is o for x in outs].index(True)
        assert not torch.equal(o, before[i])
