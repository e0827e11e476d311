"""Helpers of the tests of the calls for heads: inputs from a seed, comparison with the float64 oracle."""
import numpy as np
import torch

from lm_helpers import DTYPES, assert_within, half_step, host, normal, tiny
from oracle import heads as oracle
from paper_1908_05033_amd import binding as B

__all__ = ["B", "DTYPES", "assert_within", "half_step", "host", "normal", "oracle", "tiny", "starts", "rotation", "qkv", "check_rope", "check_prompt",
           "operand_tiny"]


def operand_tiny(dtype):
    """Half the distance of the smallest numbers, of an operand of a product: bfloat16 and binary32 have none that matter."""
    return 2.0 ** -25 if dtype == torch.float16 else 0.0


def starts(*sizes, first=0):
    return torch.tensor(np.concatenate([[0], np.cumsum(sizes)]) + first, dtype=torch.int32, device="cuda")


def rotation(seed, rows, rope_dim, axes=1, far=40000):
    """positions, pair_axis, frequencies."""
    rs = np.random.RandomState(seed)
    pairs = rope_dim // 2
    positions = torch.tensor(rs.randint(-far if seed % 2 else 0, far, (axes, rows)), dtype=torch.int32, device="cuda")
    axis = torch.tensor(rs.randint(0, axes, pairs), dtype=torch.uint8, device="cuda") if axes > 1 else None
    return positions, axis, torch.tensor(1e4 ** -(np.arange(pairs) / max(1, pairs)), dtype=torch.float32, device="cuda")


def qkv(seed, rows, hq, hk, dim, dtype, scale=1.0):
    """Parts of one tensor."""
    t = normal(seed, rows, hq + 2 * hk, dim, dtype=dtype, scale=scale)
    return t[:, :hq], t[:, hq:hq + hk], t[:, hq + hk:]


def check_rope(x, weight, eps, turning, interleaved, got, what):
    angle = oracle.angles(host(turning[0]).astype(np.int64), None if turning[1] is None else turning[1].cpu().numpy(), host(turning[2]))
    want, bound = oracle.norm_rope(host(x), None if weight is None else host(weight), eps, angle, interleaved)
    assert_within(host(got), want, bound + half_step(x.dtype) * (np.abs(want) + bound) + tiny(x.dtype), what)


def check_prompt(q, k, v, q_at, k_at, causal, scale, out, lse=None, grad=None, grads=None, left=None):
    """All results of a packed call against the oracle; q_at and k_at are the starts on the host.  `left`: what rows of no sequence hold."""
    dt, group = q.dtype, q.shape[1] // k.shape[1]
    half = half_step(dt)
    hq, hk, hv, ho = (host(t) for t in (q, k, v, out))
    hg = None if grad is None else host(grad)
    hgrads = None if grads is None else [host(t) for t in grads]
    hl = None if lse is None else host(lse)
    rounded = lambda pair: (pair[0], pair[1] + half * (np.abs(pair[0]) + pair[1]) + tiny(dt))
    for s in range(len(q_at) - 1):
        a, b, c, d = q_at[s], q_at[s + 1], k_at[s], k_at[s + 1]
        seen = oracle.causal(b - a, d - c) if causal else np.ones((b - a, d - c), bool)
        for kv in range(k.shape[1]):
            dk, dv = [], []
            for h in range(kv * group, (kv + 1) * group):
                r = oracle.attention(hq[a:b, h], hk[c:d, kv], hv[c:d, kv], seen, scale, half, None if grad is None else hg[a:b, h], operand_tiny(dt))
                what = "sequence %d head %d " % (s, h)
                assert_within(ho[a:b, h], *rounded(r["out"]), what + "out")
                if lse is not None:
                    none = np.isneginf(r["lse"][0])
                    assert np.array_equal(np.isneginf(hl[h, a:b]), none), what + "lse"
                    assert_within(hl[h, a:b][~none], r["lse"][0][~none], r["lse"][1][~none], what + "lse")
                if grad is not None:
                    assert_within(hgrads[0][a:b, h], *rounded(r["dq"]), what + "grad_q")
                    dk.append(r["dk"])
                    dv.append(r["dv"])
            if grad is not None:
                for name, got, parts in (("grad_k", hgrads[1], dk), ("grad_v", hgrads[2], dv)):
                    pair = (sum(p[0] for p in parts), sum(p[1] for p in parts) + 4 * group * oracle.U * sum(np.abs(p[0]) for p in parts))
                    assert_within(got[c:d, kv], *rounded(pair), "sequence %d key head %d %s" % (s, kv, name))
    if left is not None:
        for t, at in ((out, q_at),) + (() if grads is None else ((grads[0], q_at), (grads[1], k_at), (grads[2], k_at))):
            assert (t[:at[0]] == left).all() and (t[at[-1]:] == left).all()
