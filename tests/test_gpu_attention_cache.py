"""Attention of single tokens and of trees of drafted tokens over a paged cache, against float64."""
import numpy as np
import pytest
import torch

from heads_helpers import B, DTYPES, assert_within, half_step, host, normal, operand_tiny, oracle, starts, tiny

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def random_tree(seed, n):
    """Masks [n, words] of a tree: a token sees itself and what it descends from."""
    rs, seen = np.random.RandomState(seed), []
    for i in range(n):
        parent = rs.randint(-1, i)
        seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
    words = max(1, -(-n // 64))
    return [[w >> 64 * j & (1 << 64) - 1 for j in range(words)] for w in seen]


class Case:
    """Sequences of `lengths` keys whose last `drafted` (a number each) are the rows.  What no sequence holds in the cache is NaN."""

    def __init__(self, seed, dtype, lengths, drafted, hq, hk, dim, page, tree=False, max_rows=None, behind=0):
        dt = self.dt = DTYPES[dtype]
        rs = np.random.RandomState(seed)
        self.lengths, self.drafted, self.hq, self.hk, self.dim, self.page = lengths, drafted, hq, hk, dim, page
        rows = sum(drafted) + behind
        self.q = normal(seed, rows, hq, dim, dtype=dt, scale=1.5)
        need = [-(-n // page) for n in lengths]
        self.pages = sum(need) + 2
        self.cache = [torch.full((self.pages, hk, page, dim), NAN, dtype=dt, device="cuda") for _ in "kv"]
        order, at, self.kv = rs.permutation(self.pages)[:sum(need)], 0, []
        self.table = torch.full((len(lengths), max(need + [1]) + 1), 2 ** 31 - 1, dtype=torch.int32)
        for s, n in enumerate(lengths):
            kv = [normal(seed + 10 * s + i, n, hk, dim, dtype=dt) for i in (1, 2)]
            self.kv.append(kv)
            ids = order[at:at + need[s]]
            at += need[s]
            self.table[s, :need[s]] = torch.tensor(ids.astype(np.int32))
            if n:
                j = torch.arange(n)
                page_of = torch.tensor(ids)[j // page].cuda()
                for cache, heads in zip(self.cache, kv):
                    cache[page_of, :, (j % page).cuda()] = heads
        self.table = self.table.cuda()
        self.n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.max_rows = max_rows or max(drafted + [1])
        self.words, self.tree = None, None
        if tree:
            w = max(1, -(-max(drafted) // 64))
            self.words = [np.array([row + [0] * (w - len(row)) for row in random_tree(seed + s, n)], dtype=np.uint64).reshape(n, w) for s, n in enumerate(drafted)]
            all_ = np.concatenate(self.words + [np.zeros((behind, w), np.uint64)])
            self.tree = torch.tensor(all_.view(np.int64), device="cuda")
        self.starts = None if drafted == [1] * len(lengths) and not behind else starts(*drafted)
        self.scale = dim ** -0.5
        self.out = torch.full(self.q.shape, 7.0, dtype=dt, device="cuda")
        self.ws = torch.full((B.dsq_attention_cache_bytes(len(lengths), self.max_rows, hq, hk, dim),), 0xFF, dtype=torch.uint8, device="cuda")

    def run(self, stream=None):
        B.dsq_attention_cache(self.q, self.starts, self.max_rows, *self.cache, self.table, self.n, self.tree, self.scale, self.out, self.ws, stream)
        return self

    def check(self, hidden=None):
        """hidden: for each sequence the keys that no row sees."""
        half, group, at = half_step(self.dt), self.hq // self.hk, 0
        q, out = host(self.q), host(self.out)
        for s, (m, n) in enumerate(zip(self.lengths, self.drafted)):
            seen = oracle.tree_mask(n, m, None if self.words is None else self.words[s])
            if hidden is not None:
                seen = seen & ~hidden[s][None]
            k, v = (host(t) for t in self.kv[s])
            live = min(n, self.max_rows)
            for h in range(self.hq):
                r = oracle.attention(q[at:at + n, h], k[:, h // group], v[:, h // group], seen, self.scale, half, tiny=operand_tiny(self.dt))
                want, bound = (t[:live] for t in r["out"])
                assert_within(out[at:at + live, h], want, bound + half * (np.abs(want) + bound) + tiny(self.dt), "sequence %d head %d" % (s, h))
            assert (out[at + live:at + n] == 7).all()
            at += n
        assert (out[at:] == 7).all()


LENGTHS = [1, 2, 15, 31, 32, 33, 64, 100, 127, 128, 129, 255, 257, 500, 1000]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", [1, 16, 32, 256])
def test_single_tokens(page, dtype):
    """Each length alone and all together, with sequences that have no key among them."""
    for n in LENGTHS:
        Case(n, dtype, [n], [1], 4, 1, 128, page).run().check()
    Case(1, dtype, LENGTHS + [0, 700, 0], [1] * (len(LENGTHS) + 3), 8, 2, 64, page).run().check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [8, 24, 40, 64, 72, 80, 96, 120, 128])
def test_dims(dim, dtype):
    Case(dim, dtype, [77, 300], [1, 1], 6, 3, dim, 16).run().check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hq,hk", [(1, 1), (8, 8), (32, 1), (40, 1), (7, 7), (12, 4), (24, 3), (128, 2)])
def test_heads(hq, hk, dtype):
    Case(hq, dtype, [200, 50], [1, 1], hq, hk, 64, 64).run().check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("drafted,lengths", [([5], [5]), ([3], [40]), ([8, 1, 0, 4], [300, 1, 9, 4]), ([33, 2], [64, 129]), ([64], [700]), ([70, 130], [70, 300]),
                                             ([20, 0, 31], [0, 50, 12]), ([16] * 5, [16, 100, 31, 250, 33])])
def test_drafted(drafted, lengths, tree, dtype):
    """Chains and trees; sequences without rows, and of fewer keys than rows; more drafted tokens than a word has bits."""
    for hq, hk, page in ((4, 1, 16), (6, 3, 64), (16, 2, 4)):
        Case(sum(drafted), dtype, lengths, drafted, hq, hk, 64, page, tree, behind=3).run().check()


@pytest.mark.parametrize("dtype", DTYPES)
def test_masks_that_leave_a_row_empty(dtype):
    c = Case(3, dtype, [6, 40], [6, 6], 4, 2, 64, 16, tree=True)
    for w in c.words:
        w[2] = 0
        w[4] = 1 << 5
    c.tree = torch.tensor(np.concatenate(c.words).view(np.int64), device="cuda")
    c.run().check()
    assert not c.out[2].any()


def test_more_rows_than_announced():
    """Rows past max_rows in their sequence are left as they were; the others see what they would."""
    Case(4, "bf16", [50, 90], [10, 4], 4, 2, 64, 16, max_rows=5).run().check()
    Case(4, "bf16", [50, 90], [10, 4], 4, 2, 64, 16, tree=True, max_rows=3).run().check()
    Case(4, "bf16", [50, 90], [10, 4], 4, 2, 64, 16, max_rows=100).run().check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", [4, 32, 64])
def test_pages_outside_the_cache(page, dtype):
    """Their keys are seen by no row; a sequence of such pages alone is zeros."""
    c = Case(5, dtype, [400, 100, 130], [2, 1, 3], 4, 2, 64, page)
    table, hidden = c.table.clone(), []
    gone = {0: ([0, 3, 5], [-1, c.pages, -2 ** 31]), 1: (list(range(-(-100 // page))), [-1] * -(-100 // page)), 2: ([1], [2 ** 31 - 1])}
    for s, n in enumerate(c.lengths):
        at, ids = gone[s]
        table[s, at] = torch.tensor(ids, dtype=torch.int32, device="cuda")
        hidden.append(np.isin(np.arange(n) // page, at))
    c.table = table
    c.run().check(hidden)
    assert not c.out[2].any()


def test_lengths_outside_the_table():
    """More than the table has pages for counts as that; less than nothing as nothing."""
    c = Case(6, "f16", [64, 48], [1, 1], 4, 2, 64, 16)
    c.table = c.table[:, :4].contiguous()
    c.n = torch.tensor([2 ** 31 - 1, -7], dtype=torch.int32, device="cuda")
    c.lengths, c.kv[1] = [64, 0], [t[:0] for t in c.kv[1]]
    c.run().check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_what_is_not_seen_has_no_part(bad, dtype):
    """Bad values in drafted tokens spoil the rows that see them and no other."""
    clean = Case(7, dtype, [300, 45], [12, 5], 4, 2, 64, 16, tree=True).run()
    clean.check()
    c = Case(7, dtype, [300, 45], [12, 5], 4, 2, 64, 16, tree=True)
    place = 300 - 12 + 1                                       # drafted key 1 of the first sequence
    id_ = int(c.table[0, place // 16])
    for t in c.cache:
        t[id_, 1, place % 16, 9] = bad
    c.run()
    sees = np.array([int(w[0]) >> 1 & 1 for w in c.words[0]], bool)
    assert sees.any() and not sees.all()
    rows = torch.zeros(17, 4, dtype=torch.bool, device="cuda")
    rows[:12, 2:] = torch.tensor(sees, device="cuda")[:, None]
    assert torch.isfinite(c.out[~rows]).all()
    far = (c.out.double() - clean.out.double()).abs()[~rows]
    assert (far <= 8 * half_step(c.dt) * clean.out.double().abs()[~rows] + 64 * half_step(c.dt)).all()
    assert torch.equal(c.out[:, :2], clean.out[:, :2]) and torch.equal(c.out[12:], clean.out[12:])
    if bad is NAN:
        assert torch.isnan(c.out[rows]).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_long_and_uneven(dtype):
    """A long sequence beside short ones: chunks of one length; scores that rise along it."""
    Case(8, dtype, [9000, 3, 700, 1], [1, 2, 1, 1], 8, 2, 128, 64).run().check()
    Case(9, dtype, [20000], [1], 8, 1, 64, 16).run().check()
    c = Case(10, dtype, [3000], [4], 4, 1, 64, 16, tree=True)
    c.q[..., 0] = 8
    for j in range(0, 3000, 16):
        id_, n = int(c.table[0, j // 16]), min(16, 3000 - j)
        rise = torch.linspace(-40 + j * 0.025, -40 + (j + n) * 0.025, n).to(c.dt).cuda()
        c.cache[0][id_, :, :n, 0] = rise
        c.kv[0][0][j:j + n, :, 0] = rise[:, None]
    c.run().check()


def test_many_sequences():
    """More than a wave looks at at once."""
    rs = np.random.RandomState(3)
    lengths = rs.randint(0, 90, 300).tolist()
    Case(11, "bf16", lengths, [1] * 300, 2, 1, 32, 16).run().check()
    drafted = [int(min(n, d)) for n, d in zip(lengths, rs.randint(0, 4, 300))]
    Case(12, "bf16", lengths, drafted, 2, 1, 32, 16, tree=True).run().check()


def test_offsets_past_32_bits():
    """A cache of more than 2^32 bytes and 2^31 elements whose last pages are used."""
    pages, hk, page, dim = 2100, 8, 1024, 128
    c = Case(13, "bf16", [1500, 300], [1, 3], 16, hk, dim, page)
    big = [torch.zeros(pages, hk, page, dim, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    assert big[0].numel() > 2 ** 31
    for b, small in zip(big, c.cache):
        b[-c.pages:] = small
    c.table = torch.where(c.table < c.pages, c.table + (pages - c.pages), c.table)
    c.cache = big
    c.run().check()


def test_rows_of_heads_and_tables_apart():
    c = Case(14, "bf16", [70, 130, 20], [2, 1, 3], 4, 2, 64, 16, tree=True)
    c.run()
    want = c.out.clone()
    c.q = c.q.transpose(0, 1).contiguous().transpose(0, 1)
    room = torch.full((4, 6, 80), 5.0, dtype=c.dt, device="cuda")
    c.out = room[:, :, 8:72].transpose(0, 1)
    wide = torch.full((3, 40), -1, dtype=torch.int32, device="cuda")
    wide[:, :c.table.shape[1]] = c.table
    c.table = wide[:, :c.table.shape[1]]
    c.run()
    assert torch.equal(c.out, want) and (room[..., :8] == 5).all() and (room[..., 72:] == 5).all()
    # one table for all: sequences that share their pages
    c = Case(15, "bf16", [100], [1], 4, 2, 64, 16)
    c.run().check()
    d = Case(16, "bf16", [100, 100], [1, 1], 4, 2, 64, 16)
    d.cache, d.kv, d.table = c.cache, c.kv * 2, c.table.expand(2, -1)
    d.run().check()


def test_same_bits_every_time():
    for dtype in DTYPES:
        c = Case(17, dtype, [3000, 70, 500], [4, 1, 9], 8, 2, 64, 16, tree=True).run()
        first = c.out.clone()
        for _ in range(3):
            c.ws.fill_(0xFF)
            assert torch.equal(c.run().out, first)


def test_nothing_to_do():
    c = Case(18, "f32", [5], [1], 2, 1, 32, 16)
    e = torch.empty(0, 2, 32, device="cuda")
    B.dsq_attention_cache(e, starts(0), 1, *c.cache, c.table, c.n, None, 1.0, e, c.ws)
    none = torch.empty(0, 1, 16, 32, device="cuda")
    B.dsq_attention_cache(c.q, None, 1, none, none, c.table, c.n, None, 1.0, c.out, c.ws)
    assert not c.out.any()
    c.out.fill_(7)
    B.dsq_attention_cache(c.q, None, 1, *c.cache, c.table[:, :0], c.n, None, 1.0, c.out, c.ws)
    assert not c.out.any()
