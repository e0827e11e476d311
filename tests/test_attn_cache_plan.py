"""The chunks that attention over a cache cuts keys into, as host arithmetic: numbers of chunks and tiles, compiled from the
headers that the library uses, against plain sums over the sequences."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text('#include "%s/paper_1908_05033_amd/csrc/attn_cache_plan.h"\n'
                                'extern "C" void plan(int m, int q, int k, int s, long long n, int *o)\n'
                                '{ AttnCachePlan p = attn_cache_plan(m, q, k, s, n); o[0] = p.tiles; o[1] = p.single; o[2] = p.row_tiles; o[3] = p.slots; }\n' % ROOT)
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-o", str(d / "plan.so"), str(d / "plan.cpp")], check=True)
    lib = ctypes.CDLL(str(d / "plan.so"))

    def call(max_rows, q_heads, kv_heads, sequences, keys):
        o = (ctypes.c_int * 4)()
        lib.plan(max_rows, q_heads, kv_heads, sequences, ctypes.c_longlong(keys), o)
        return dict(tiles=bool(o[0]), single=bool(o[1]), row_tiles=o[2], slots=o[3])
    return call


def test_plan(plan):
    assert plan(1, 32, 8, 1, 512) == dict(tiles=False, single=True, row_tiles=1, slots=0)
    assert plan(1, 32, 8, 1, 4096) == dict(tiles=False, single=False, row_tiles=1, slots=64)
    assert plan(1, 32, 8, 2, 4096)["slots"] == 128
    assert plan(48, 32, 8, 8, 512) == dict(tiles=True, single=False, row_tiles=2, slots=32)
    assert plan(8, 32, 8, 1, 4096)["tiles"] is False and plan(9, 32, 8, 1, 4096)["tiles"] is True
    assert plan(1 << 20, 1024, 1, 1, 1 << 30)["slots"] == 1
    for rows in (1, 3, 40):
        for heads in ((1, 1), (64, 8), (1024, 1024)):
            p = plan(rows, *heads, 5, 1 << 20)
            assert p["slots"] >= 1 and p["row_tiles"] >= 1 and not p["single"]


def chunks(lengths, slots):
    """What the kernels do: units a chunk, and the first number of each sequence."""
    units = [-(-n // 128) for n in lengths]
    per = max(1, -(-sum(units) // slots))
    before = np.concatenate([[0], np.cumsum(units)])[:-1]
    return per, [int(b // per + s) for s, b in enumerate(before)], [-(-u // per) for u in units]


def test_numbers_of_chunks_do_not_meet():
    """Each sequence has room for its chunks before the next one's first number, and all numbers are below slots + sequences."""
    rs = np.random.RandomState(1)
    for _ in range(300):
        n, slots = rs.randint(1, 70), rs.choice([1, 2, 7, 64, 128])
        lengths = (rs.randint(0, 2, n) * 10 ** rs.uniform(0, 5, n)).astype(int).tolist()
        per, first, count = chunks(lengths, slots)
        ends = [f + max(1, c) for f, c in zip(first, count)]
        assert all(e <= f for e, f in zip(ends, first[1:])) and ends[-1] <= slots + n


def test_numbers_of_tiles_do_not_meet():
    """Tiles of packed sequences: starts[s] / tile + s is room for all tiles of the sequences before."""
    rs = np.random.RandomState(2)
    for _ in range(300):
        n, tile = rs.randint(1, 50), rs.choice([32, 64, 128])
        starts = np.concatenate([[0], np.cumsum(rs.randint(0, 2, n) * rs.randint(0, 500, n))]) + rs.randint(0, 200)
        first = starts // tile + np.arange(n + 1)
        need = -(-np.diff(starts) // tile)
        assert (first[:-1] + need <= first[1:]).all() and first[-1] <= starts[-1] // tile + n
