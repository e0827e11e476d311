"""The language-model calls together, as a program uses them: a block of serving calls and a training step, eager, on another
stream, in captured graphs, and by both ways of the binding."""
import numpy as np
import pytest
import torch

from oracle import lm
from paper_1908_05033_amd import binding as B
from lm_helpers import DTYPES, U32, assert_within, host, normal, pack, random_w4
from test_gpu_rms_norm import check_bwd, check_fwd
from test_gpu_w4 import check

pytestmark = pytest.mark.gpu
EPS = 1e-5


class Serving:
    """x + residual -> norm -> 8-bit rows -> layer of 4-bit weights -> + sum -> norm -> float rows -> layer."""

    def __init__(self, M, dim, wide, dt, group=64, seed=1):
        self.M, self.dim, self.wide, self.group, self.dt = M, dim, wide, group, dt
        e = lambda *s, **k: torch.empty(*s, device="cuda", **{"dtype": dt, **k})
        self.x, self.res = normal(seed, M, dim, dtype=dt), normal(seed + 1, M, dim, dtype=dt, scale=2.0)
        self.w1, self.w2 = normal(seed + 2, dim, dtype=dt), normal(seed + 3, dim, dtype=dt)
        self.l1, self.l2 = random_w4(seed, dim, dim, group), random_w4(seed + 1, wide, dim, group)
        self.p1, self.p2 = pack(*self.l1, group), pack(*self.l2, group)
        self.bias = normal(seed + 4, wide, dtype=dt)
        self.h1, self.h2, self.a, self.y, self.out = e(M, dim), e(M, dim), e(M, dim), e(M, dim), e(M, wide)
        self.q, self.qs = e(M, B.dsq_code_row_bytes(dim), dtype=torch.int8), e(M, dtype=torch.float32)

    def run(self, stream=None):
        B.dsq_rms_norm(self.x, self.res, self.w1, EPS, self.h1, None, self.q, self.qs, None, stream)
        B.dsq_linear_w4a8(self.q, self.qs, *self.p1, self.dim, self.dim, self.group, None, self.a, stream)
        B.dsq_rms_norm(self.a, self.h1, self.w2, EPS, self.h2, self.y, None, None, None, stream)
        B.dsq_linear_w4(self.y, *self.p2, self.wide, self.dim, self.group, self.bias, self.out, stream)

    def results(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.h1, self.q, self.qs, self.a, self.h2, self.y, self.out)]

    def scramble(self):
        for t in (self.h1, self.a, self.h2, self.y, self.out, self.qs):
            t.fill_(float("nan"))
        self.q.fill_(55)

    def check(self):
        first = {"sum": self.h1, "y": None, "rstd": None, "codes": self.q, "scales": self.qs}
        check_fwd(self.x, self.res, self.w1, first, EPS)
        check(self.a, host(self.q[:, :self.dim]) * host(self.qs)[:, None], *self.l1, self.group, ints=True)
        second = {"sum": self.h2, "y": self.y, "rstd": None, "codes": None}
        check_fwd(self.a, self.h1, self.w2, second, EPS)
        check(self.out, host(self.y), *self.l2, self.group, self.bias)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", [1, 2, 13, 40, 300])
def test_serving(M, dtype):
    for dim, wide in ((384, 1000), (1001, 70)):
        s = Serving(M, dim, wide, DTYPES[dtype])
        s.run()
        torch.cuda.synchronize()
        s.check()


@pytest.mark.parametrize("M", [1, 9, 150])
def test_serving_in_graphs_and_on_other_streams(M):
    a, b = Serving(M, 520, 300, torch.bfloat16), Serving(M, 520, 300, torch.bfloat16, seed=50)
    a.run()
    b.run()
    want_a, want_b = a.results(), b.results()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    # the stream given by its object and by its handle, the current one being another
    for t in (s1, s2.cuda_stream):
        a.scramble()
        torch.cuda.synchronize()
        a.run(t)
        assert all(torch.equal(x, y) for x, y in zip(a.results(), want_a))
    # two at once
    a.scramble(), b.scramble()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(s1):
            a.run()
        with torch.cuda.stream(s2):
            b.run()
    assert all(torch.equal(x, y) for x, y in zip(a.results() + b.results(), want_a + want_b))
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
        assert all(torch.equal(x, y) for x, y in zip(a.results() + b.results(), want_a + want_b))
        a.run()                                             # eager work between the replays
        assert all(torch.equal(x, y) for x, y in zip(a.results(), want_a))
    # new inputs in the same places
    a.x.copy_(normal(77, M, 520, dtype=torch.bfloat16))
    graphs[0].replay()
    torch.cuda.synchronize()
    a.check()


class Training:
    """Two norms along a residual stream and their backward passes:  h1 = x + residual, y1 = norm(h1), h2 = y1 + h1,
    y2 = norm(h2), a gradient arrives at y2 and at h2."""

    def __init__(self, rows, dim, dt, seed=1):
        e = lambda *s, **k: torch.empty(*s, device="cuda", **{"dtype": dt, **k})
        self.x, self.res = normal(seed, rows, dim, dtype=dt), normal(seed + 1, rows, dim, dtype=dt)
        self.w1, self.w2 = normal(seed + 2, dim, dtype=dt), normal(seed + 3, dim, dtype=dt)
        self.gy, self.gs = normal(seed + 4, rows, dim, dtype=dt), normal(seed + 5, rows, dim, dtype=dt)
        self.h1, self.y1, self.h2, self.y2, self.gh2, self.gx = (e(rows, dim) for _ in range(6))
        self.r1, self.r2 = e(rows, dtype=torch.float32), e(rows, dtype=torch.float32)
        self.gw1, self.gw2 = e(dim, dtype=torch.float32), e(dim, dtype=torch.float32)
        self.ws = e(B.dsq_rms_norm_bwd_bytes(rows, dim), dtype=torch.uint8)

    def run(self):
        B.dsq_rms_norm(self.x, self.res, self.w1, EPS, self.h1, self.y1, None, None, self.r1)
        B.dsq_rms_norm(self.y1, self.h1, self.w2, EPS, self.h2, self.y2, None, None, self.r2)
        # (one workspace for calls that follow one another)
        B.dsq_rms_norm_bwd(self.h2, self.w2, self.r2, self.gy, self.gs, self.gh2, self.gw2, self.ws)
        B.dsq_rms_norm_bwd(self.h1, self.w1, self.r1, self.gh2, self.gh2, self.gx, self.gw1, self.ws)

    def results(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.h1, self.y1, self.h2, self.y2, self.gh2, self.gx, self.gw1, self.gw2)]

    def scramble(self):
        for t in (self.h1, self.y1, self.h2, self.y2, self.gh2, self.gx, self.gw1, self.gw2, self.r1, self.r2):
            t.fill_(float("nan"))
        self.ws.fill_(0xFF)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,dim", [(1, 96), (50, 515), (700, 256), (20, 9001)])
def test_training(rows, dim, dtype):
    t = Training(rows, dim, DTYPES[dtype])
    t.run()
    check_bwd(t.h2, t.w2, t.r2, t.gy, t.gs, t.gh2, t.gw2)
    check_bwd(t.h1, t.w1, t.r1, t.gh2, t.gh2, t.gx, t.gw1)


def test_training_against_differences():
    """Both norms' gradients against central differences of the float64 oracle: every step of the chain rounds to binary32,
    gradients of six values a number at most, as in the test of one norm."""
    t = Training(6, 515, torch.float32)
    t.run()
    torch.cuda.synchronize()
    x, res, w1, w2, gy, gs = (host(v) for v in (t.x, t.res, t.w1, t.w2, t.gy, t.gs))

    def loss(a, u, v):
        h1 = a + res
        h2 = lm.rms_norm(h1, u, EPS)[0] + h1
        return (gy * lm.rms_norm(h2, v, EPS)[0]).sum() + (gs * h2).sum()

    rs, step = np.random.RandomState(3), 1e-6
    for got, at in ((t.gx, 0), (t.gw1, 1), (t.gw2, 2)):
        for _ in range(4):
            d = rs.randn(*got.shape)
            up, down = [x, w1, w2], [x, w1, w2]
            up[at], down[at] = up[at] + step * d, down[at] - step * d
            diff = (loss(*up) - loss(*down)) / (2 * step)
            assert abs(diff - (host(got) * d).sum()) <= 1e-5 * np.abs(host(got) * d).sum()


@pytest.mark.parametrize("rows,dim", [(3, 96), (1500, 520)])
def test_training_in_graphs(rows, dim):
    """Two captured steps with a workspace each, replayed at once, and an eager one with its own between."""
    a, b = Training(rows, dim, torch.bfloat16), Training(rows, dim, torch.bfloat16, seed=50)
    a.run()
    b.run()
    want_a, want_b = a.results(), b.results()
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
        b.run()
        assert all(torch.equal(x, y) for x, y in zip(b.results(), want_b))


def test_empty_gradient_in_a_graph():
    """No rows: the weight's gradient is zeros, in a replay too."""
    e, gw = torch.empty(0, 700, device="cuda"), torch.full((700,), 3.0, device="cuda")
    r = torch.empty(0, device="cuda")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            B.dsq_rms_norm_bwd(e, None, r, e, None, e, gw, None)
        for _ in range(3):
            gw.fill_(5.0)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert not gw.any()


class General:
    """A marshalling module that leaves every call to the general path."""

    def __getattr__(self, name):
        return lambda *a: None


def test_both_ways_of_the_binding(monkeypatch):
    runs = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(B, "_marshal", General())
        s, t = Serving(7, 392, 100, torch.float16), Training(9, 264, torch.float32)
        s.run()
        t.run()
        wide = normal(3, 7, 500, dtype=torch.float16)[:, 8:400]
        out = torch.zeros(7, 130, dtype=torch.float16, device="cuda")
        B.dsq_linear_w4(wide, *s.p2, s.wide, s.dim, s.group, None, out[:, :100], torch.cuda.current_stream())
        runs.append(s.results() + t.results() + [out.clone()])
    assert all(torch.equal(x, y) for x, y in zip(*runs))


@pytest.mark.parametrize("native", [True, False])
def test_refusals(native, monkeypatch):
    if not native:
        monkeypatch.setattr(B, "_marshal", General())
    s, t = Serving(4, 256, 64, torch.bfloat16), Training(4, 64, torch.float32)
    before = s.results()
    norm = lambda x=s.x, res=s.res, w=s.w1, eps=EPS, h=s.h1, y=None, q=s.q, qs=s.qs, r=None: B.dsq_rms_norm(x, res, w, eps, h, y, q, qs, r)
    lin = lambda x=s.y, w=s.p2[0], sc=s.p2[1], N=64, K=256, g=64, b=s.bias, o=s.out: B.dsq_linear_w4(x, w, sc, N, K, g, b, o)
    lin8 = lambda q=s.q, qs=s.qs, w=s.p1[0], sc=s.p1[1], N=256, K=256, g=64, b=None, o=s.a: B.dsq_linear_w4a8(q, qs, w, sc, N, K, g, b, o)
    bwd = lambda h=t.x, w=t.w1, r=t.r1, gy=t.gy, gs=t.gs, gx=t.gx, gw=t.gw1, ws=t.ws: B.dsq_rms_norm_bwd(h, w, r, gy, gs, gx, gw, ws)
    f32 = lambda v: v.float()
    for call, status in ((lambda: norm(res=s.res[:2]), 4), (lambda: norm(w=s.w1[:64]), 4), (lambda: norm(h=s.h1[:3]), 4),
                         (lambda: norm(q=s.q[:, :128]), 4), (lambda: norm(qs=s.qs[:3]), 4), (lambda: norm(qs=None), 1), (lambda: norm(q=None), 1),
                         (lambda: norm(eps=0.0), 3), (lambda: norm(eps=float("nan")), 3), (lambda: norm(x=None), 1),
                         (lambda: norm(x=s.x[0]), 4), (lambda: norm(h=None, q=None, qs=None), 1),
                         (lambda: lin(N=63), 4), (lambda: lin(K=255), 4), (lambda: lin(g=48), 5), (lambda: lin(N=4096, o=torch.empty(4, 4096, dtype=s.dt, device="cuda"), b=None), 7),
                         (lambda: lin(g=32), 7), (lambda: lin(o=s.out[:3]), 4), (lambda: lin(b=s.bias[:32]), 4), (lambda: lin(w=s.p2[0][:64]), 7),
                         (lambda: lin(o=torch.empty(1, 64, dtype=s.dt, device="cuda").expand(4, 64)), 4),
                         (lambda: lin8(K=300), 4), (lambda: lin8(qs=s.qs[:1]), 4), (lambda: lin8(N=255), 4), (lambda: lin8(sc=s.p1[1][:128]), 7),
                         (lambda: bwd(r=t.r1[:2]), 4), (lambda: bwd(gy=t.gy[:, :32]), 4), (lambda: bwd(ws=t.ws[:16]), 7), (lambda: bwd(ws=None), 1),
                         (lambda: bwd(gx=None), 1), (lambda: bwd(gw=t.gw1[:32]), 4)):
        with pytest.raises(B.DsqError) as e:
            call()
        assert e.value.status == status, (status, str(e.value))
    for call in (lambda: norm(res=f32(s.res)), lambda: norm(w=f32(s.w1)), lambda: norm(x=s.x.double()), lambda: norm(x=s.x.cpu()),
                 lambda: norm(q=s.q.view(torch.uint8)), lambda: norm(x=normal(1, 256, 4, dtype=s.dt).t()), lambda: norm(h=torch.empty(4, 300, dtype=s.dt, device="cuda")[:, :256]),
                 lambda: lin(b=f32(s.bias)), lambda: lin(o=f32(s.out)), lambda: lin(x=s.y.to(torch.int8)), lambda: lin(w=s.p2[0].view(torch.int8)),
                 lambda: lin(o=torch.empty(64, 4, dtype=s.dt, device="cuda").t()), lambda: lin8(q=s.q.float()), lambda: lin8(qs=s.qs.double()),
                 lambda: lin8(o=s.a.to(torch.int32)), lambda: bwd(gs=t.gs.half()), lambda: bwd(gw=t.gw1.half())):
        with pytest.raises(TypeError):
            call()
    # (an address that is no multiple of 16)
    with pytest.raises(B.DsqError) as e:
        norm(x=torch.empty(4 * 256 + 1, dtype=s.dt, device="cuda")[1:].view(4, 256))
    assert e.value.status == 6
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(s.results(), before) if not a.is_floating_point())
