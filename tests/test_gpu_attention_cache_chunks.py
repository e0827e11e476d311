"""Attention over a paged cache in chunks of several blocks of keys a wave, and all kernels that join them, against float64.  test_attn_cache_numbers.py
holds that these shapes have such chunks and take those kernels."""
import numpy as np
import pytest
import torch

from heads_helpers import B, DTYPES, half_step
from lm_helpers import U32
from test_gpu_attention_cache import Case

pytestmark = pytest.mark.gpu

MANY = np.random.RandomState(1).randint(0, 1500, 80).tolist()
# name: lengths, drafted tokens, query heads, key heads, elements, page, tree
SHAPES = {
    "tokens": ([9000, 5001, 300], [1, 1, 1], 64, 64, 32, 16, False),
    "one long": ([20000], [1], 32, 16, 64, 64, False),
    "wide heads": ([7000, 4100], [2, 1], 24, 24, 128, 256, False),
    # a chunk has 512 keys
    "ends": ([511, 512, 513, 1023, 1024, 1025, 1536, 4000, 5500, 127, 1, 0], [1] * 12, 64, 32, 40, 16, False),
    "short trees": ([9000, 5000, 300], [16, 16, 16], 90, 45, 32, 32, True),
    "trees": ([6000, 3001, 100, 2048], [40, 3, 17, 40], 32, 16, 64, 64, True),
    # a chunk of 384 keys, small pages
    "trees' ends": ([383, 384, 385, 769, 3000, 2690], [20, 33, 1, 0, 40, 40], 40, 20, 72, 16, True),
    "two tiles": ([5000, 2500, 384], [70, 70, 5], 30, 15, 128, 128, True),
    "many": (MANY, [1] * 80, 16, 8, 32, 16, False),
    "many drafted": (MANY, [i % 4 for i in range(80)], 16, 8, 32, 16, True),
}


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", SHAPES)
def test_shapes(name, dtype):
    c = Case(len(name), dtype, *SHAPES[name])
    c.run().check()
    first = c.out.clone()
    c.ws.fill_(0xFF)
    assert torch.equal(c.run().out, first)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", ["tokens", "ends", "short trees", "trees", "trees' ends"])
def test_pages_outside_the_cache(name, dtype):
    """Pages in the middle of a chunk, its first and its last one; a whole chunk of them."""
    c = Case(3, dtype, *SHAPES[name])
    rs, hidden = np.random.RandomState(4), []
    table = c.table.clone()
    for s, n in enumerate(c.lengths):
        pages = -(-n // c.page)
        gone = np.zeros(pages, bool)
        if pages > 3:
            gone[rs.permutation(pages)[:pages // 5 + 1]] = True
            gone[pages // 3:pages // 3 + 1024 // c.page] = True
            # (the drafted tokens' own keys stay, so that no row is empty by chance alone)
            gone[pages - (-(-max(1, c.drafted[s]) // c.page) + 1):] = False
        table[s, np.flatnonzero(gone)] = torch.tensor(rs.choice([-1, c.pages, 2 ** 31 - 1, -2 ** 31], gone.sum()), dtype=torch.int32, device="cuda")
        hidden.append(gone[np.arange(n) // c.page])
    c.table = table
    c.run().check(hidden)


@pytest.mark.parametrize("dtype", DTYPES)
def test_rising_scores(dtype):
    """Scores that rise or fall along the keys, within chunks and over them: every join weighs its parts."""
    for up in (1, -1):
        for name in ("tokens", "trees"):
            c = Case(5, dtype, *SHAPES[name])
            c.q[..., 0] = 8
            for s, n in enumerate(c.lengths):
                rise = (torch.linspace(-40, 40, n) * up).to(c.dt).cuda()
                place = torch.arange(n, device="cuda")
                page = c.table[s].long()[place // c.page]
                c.cache[0][page, :, place % c.page, 0] = rise[:, None]
                c.kv[s][0][:, :, 0] = rise[:, None]
            c.run().check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", ["two tiles", "short trees"])
def test_heads_that_are_no_multiple_of_four(name, dtype):
    """A wave that joins four heads has fewer at the end of a row: what lies behind the row stays."""
    c = Case(6, dtype, *SHAPES[name])
    want = c.run().out.clone()
    c.check()
    room = torch.full((c.q.shape[0], c.hq + 3, c.dim), 5.0, dtype=c.dt, device="cuda")
    c.out = room[:, :c.hq]
    c.run()
    assert torch.equal(c.out, want) and (room[:, c.hq:] == 5).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["one long", "tokens", "trees", "short trees", "two tiles"])
def test_values_near_the_end_of_binary32(name, dtype):
    """Chunks whose weighted sum would pass binary32 before it is divided; the result, a mean of equal values, is one of them."""
    c = Case(7, dtype, *SHAPES[name])
    c.cache[1].copy_(torch.where(torch.isnan(c.cache[1]), c.cache[1], 3e38))
    c.run()
    big = float(torch.tensor(3e38, dtype=c.dt))
    # probabilities and their sum round (as in the bounds of the oracle: 4 half steps of binary32 a key), a result once
    assert ((c.out.double() / big - 1).abs() <= 2 * half_step(c.dt) + 4 * (max(c.lengths) + 16) * U32).all()
