"""Refused language-model calls leave every output as it was, floats among them: outputs are filled with numbers first."""
import pytest
import torch

from paper_1908_05033_amd import binding as B
from test_gpu_lm_layers import EPS, General, Serving, Training

pytestmark = pytest.mark.gpu


def outputs(s, t):
    return [s.h1, s.h2, s.a, s.y, s.out, s.q, s.qs, t.h1, t.y1, t.h2, t.y2, t.gh2, t.gx, t.r1, t.r2, t.gw1, t.gw2, t.ws, *s.p1, *s.p2]


@pytest.mark.parametrize("native", [True, False])
def test_refused_calls_write_nothing(native, monkeypatch):
    s, t = Serving(4, 256, 64, torch.bfloat16), Training(4, 64, torch.float32)
    torch.cuda.synchronize()
    if not native:
        monkeypatch.setattr(B, "_marshal", General())
    outs = outputs(s, t)
    for i, o in enumerate(outs):
        o.fill_(i + 3)
    before = [o.clone() for o in outs]
    norm = lambda x=s.x, res=s.res, w=s.w1, eps=EPS, h=s.h1, y=s.y, q=s.q, qs=s.qs, r=t.r1: B.dsq_rms_norm(x, res, w, eps, h, y, q, qs, r)
    lin = lambda x=s.x, w=s.p2[0], sc=s.p2[1], N=64, K=256, g=64, b=s.bias, o=s.out: B.dsq_linear_w4(x, w, sc, N, K, g, b, o)
    lin8 = lambda q=s.q, qs=s.qs, w=s.p1[0], sc=s.p1[1], N=256, K=256, g=64, b=None, o=s.a: B.dsq_linear_w4a8(q, qs, w, sc, N, K, g, b, o)
    bwd = lambda h=t.x, w=t.w1, r=t.r1, gy=t.gy, gs=t.gs, gx=t.gx, gw=t.gw1, ws=t.ws: B.dsq_rms_norm_bwd(h, w, r, gy, gs, gx, gw, ws)
    pack = lambda w=torch.ones(64, 256, device="cuda"), N=64, K=256, g=64, wp=s.p2[0], sp=s.p2[1]: B.dsq_pack_weights_w4(w, None, None, None, N, K, g, wp, sp)
    odd = torch.empty(4 * 256 + 1, dtype=s.dt, device="cuda")[1:].view(4, 256)
    for call in (lambda: norm(res=s.res[:2]), lambda: norm(w=s.w1[:64]), lambda: norm(q=s.q[:, :128]), lambda: norm(qs=s.qs[:3]),
                 lambda: norm(qs=None), lambda: norm(q=None), lambda: norm(eps=0.0), lambda: norm(eps=float("nan")), lambda: norm(x=odd),
                 lambda: norm(x=s.x.double()), lambda: norm(res=s.res.float()), lambda: norm(r=t.r1[:2]), lambda: norm(y=s.y.float()),
                 lambda: lin(N=63), lambda: lin(K=255), lambda: lin(g=48), lambda: lin(g=32), lambda: lin(b=s.bias[:32]), lambda: lin(b=s.bias.float()),
                 lambda: lin(w=s.p2[0][:64]), lambda: lin(o=s.out[:3]), lambda: lin(x=odd), lambda: lin(x=s.x.float()),
                 lambda: lin8(K=300), lambda: lin8(qs=s.qs[:1]), lambda: lin8(N=255), lambda: lin8(sc=s.p1[1][:128]), lambda: lin8(qs=s.qs.double()),
                 lambda: lin8(q=s.q.float()), lambda: lin8(g=32),
                 lambda: bwd(r=t.r1[:2]), lambda: bwd(gy=t.gy[:, :32]), lambda: bwd(ws=t.ws[:16]), lambda: bwd(ws=None), lambda: bwd(gw=t.gw1[:32]),
                 lambda: bwd(gs=t.gs.half()), lambda: bwd(h=t.x.half()),
                 lambda: pack(g=48), lambda: pack(N=63), lambda: pack(K=0), lambda: pack(wp=s.p2[0][:64]), lambda: pack(sp=s.p2[1][:64]),
                 lambda: pack(w=torch.ones(64, 256, dtype=torch.float16, device="cuda"))):
        with pytest.raises((B.DsqError, TypeError)):
            call()
    torch.cuda.synchronize()
    for i, (o, want) in enumerate(zip(outs, before)):
        assert torch.equal(o, want), i
    # (the same calls with their own arguments do write)
    norm(), lin(), lin8(), bwd(), pack()
    torch.cuda.synchronize()
    for o, want in ((s.h1, before[0]), (s.y, before[3]), (s.out, before[4]), (s.a, before[2]), (t.gx, before[12]), (t.gw1, before[15])):
        assert not torch.equal(o, want)
