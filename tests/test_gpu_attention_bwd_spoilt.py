"""Gradients beside infinities and NaN: those of every other sequence are the same to the bit, and no row of no sequence is written."""
import pytest
import torch

from heads_helpers import DTYPES
from test_gpu_attention import call

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
# sizes of the sequences, query heads, key heads: waves that split the keys (and keys' sums split over workgroups), and 128 rows a workgroup
KINDS = {"few": ([70, 130, 1, 64, 300], 4, 2), "many": ([270, 130, 1, 64, 600], 48, 4)}
SPOILT = 1


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [40, 64, 80, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind", KINDS)
def test_other_sequences_are_as_without(kind, causal, dim, dtype):
    sizes, hq, hk = KINDS[kind]
    clean = call(9, dtype, sizes, sizes, hq, hk, dim, causal, first=3, behind=70).forward().backward()
    clean.check() if kind == "few" and dim == 64 else None
    at = [3 + sum(sizes[:i]) for i in range(len(sizes) + 1)]
    a, b = at[SPOILT], at[SPOILT + 1]
    others = torch.ones(len(clean.q), dtype=torch.bool, device="cuda")
    others[a:b] = False
    for bad in (NAN, INF):
        for which in ("q", "k", "v", "grad"):
            c = call(9, dtype, sizes, sizes, hq, hk, dim, causal, first=3, behind=70)
            x = getattr(c, which).contiguous().clone()
            x[a + 5, 1, 2] = x[b - 1, 0, dim - 1] = bad
            setattr(c, which, x)
            c.forward().backward()
            assert torch.equal(c.out[others], clean.out[others]) and torch.equal(c.lse[:, others], clean.lse[:, others])
            for got, want in zip(c.grads, clean.grads):
                assert torch.equal(got[others], want[others]), (which, bad)
            assert not all(torch.isfinite(g[a:b]).all() for g in c.grads), (which, bad)
