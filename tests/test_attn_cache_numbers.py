"""How the keys of a cache are cut into chunks, compiled from the header that the library uses: no two sequences have a number in common, every key is in one
chunk, and which kernels a call takes."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import test_gpu_attention_cache_chunks as shapes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NONE, SIXTEEN, ONE, FOUR = range(4)
SOURCE = """#include "%s/paper_1908_05033_amd/csrc/attn_cache_plan.h"
extern "C" {
int units(int length) { return attn_units(length); }
int chunk_units(int total, int slots) { return attn_chunk_units(total, slots); }
int first_chunk(int before, int units, int s) { return attn_first_chunk(before, units, s); }
int chunk_keys(int units) { return attn_chunk_keys(units); }
void plan(int rows, int most, int q, int k, int s, long long n, int *o)
{
    const AttnCachePlan p = attn_cache_plan(most, q, k, s, n);
    o[0] = p.tiles; o[1] = p.single; o[2] = p.row_tiles; o[3] = p.slots; o[4] = attn_cache_join(p, rows, q, s);
}
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SOURCE % ROOT)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", str(d / "plan.so"), str(d / "plan.cpp")], check=True)
    return ctypes.CDLL(str(d / "plan.so"))


def plan(lib, rows, most, q_heads, kv_heads, sequences, keys):
    o = (ctypes.c_int * 5)()
    lib.plan(rows, most, q_heads, kv_heads, sequences, ctypes.c_longlong(keys), o)
    return dict(tiles=bool(o[0]), single=bool(o[1]), row_tiles=o[2], slots=o[3], join=o[4])


def cut(lib, lengths, slots):
    """Units a chunk, first numbers and numbers of chunks."""
    units = [lib.units(n) for n in lengths]
    per = lib.chunk_units(sum(units), slots)
    before = np.concatenate([[0], np.cumsum(units)])
    keys = lib.chunk_keys(per)
    return per, [lib.first_chunk(int(b), per, s) for s, b in enumerate(before[:-1])], [-(-n // keys) for n in lengths]


def test_numbers_of_chunks(lib):
    rs = np.random.RandomState(1)
    for _ in range(400):
        n, slots = rs.randint(1, 90), int(rs.choice([1, 2, 7, 64, 128, 512]))
        lengths = (rs.randint(0, 2, n) * 10 ** rs.uniform(0, 6, n)).astype(int).tolist()
        per, first, count = cut(lib, lengths, slots)
        # (a sequence without keys has a number all the same: its rows are zeros)
        ends = [f + max(1, c) for f, c in zip(first, count)]
        assert per >= 1 and all(e <= f for e, f in zip(ends, first[1:])) and ends[-1] <= slots + n


def test_ends_of_the_range(lib):
    assert [lib.units(n) for n in (0, 1, 128, 129, 1 << 30)] == [0, 1, 1, 2, 1 << 23]
    assert lib.chunk_units(0, 512) == 1 and lib.chunk_units(512, 512) == 1 and lib.chunk_units(513, 512) == 2 and lib.chunk_units(1 << 30, 1) == 1 << 30
    assert lib.chunk_keys(1) == 128 and lib.chunk_keys(1 << 23) == 1 << 30 and lib.chunk_keys(1 << 30) == 1 << 30
    per, first, count = cut(lib, [1 << 30] * 100, 1)
    assert count == [1] * 100 and first == sorted(set(first)) and first[-1] < 101


def of_shape(lib, name):
    lengths, drafted, hq, hk, _, page, _ = shapes.SHAPES[name]
    keys = (max(-(-n // page) for n in lengths) + 1) * page              # (of the test's table)
    p = plan(lib, sum(drafted), max(drafted), hq, hk, len(lengths), keys)
    assert not p["single"]
    return p, cut(lib, lengths, p["slots"])


def test_shapes_have_long_chunks(lib):
    """Several units a chunk, and sequences of several chunks, in each of them."""
    seen = set()
    for name, (lengths, *_) in shapes.SHAPES.items():
        p, (per, _, count) = of_shape(lib, name)
        assert per > 1 and max(count) > 1, name
        seen.add((p["tiles"], p["join"]))
    # both kernels, joined by each of the three
    assert {j for _, j in seen} == {SIXTEEN, ONE, FOUR} and {t for t, _ in seen} == {False, True}
    assert {(False, FOUR), (True, FOUR), (True, ONE), (False, ONE)} <= seen
    for name in ("short trees", "two tiles"):
        assert of_shape(lib, name)[0]["join"] == FOUR and shapes.SHAPES[name][2] % 4
    assert of_shape(lib, "two tiles")[0]["row_tiles"] == 2 and len(shapes.SHAPES["many"][0]) > 64
    for name, keys in (("ends", 512), ("trees' ends", 384)):
        assert lib.chunk_keys(of_shape(lib, name)[1][0]) == keys
        assert {keys - 1, keys, keys + 1} <= set(shapes.SHAPES[name][0])


def test_joins(lib):
    assert plan(lib, 1, 1, 32, 8, 1, 1024)["join"] == NONE and plan(lib, 1, 1, 32, 8, 1, 1025)["join"] == SIXTEEN
    assert plan(lib, 32, 32, 32, 32, 1, 8192)["join"] == SIXTEEN and plan(lib, 33, 33, 32, 32, 1, 8192)["join"] == ONE
    assert plan(lib, 4, 1, 32, 8, 4, 8192)["join"] == SIXTEEN and plan(lib, 8, 1, 32, 8, 8, 8192)["join"] == SIXTEEN
    assert plan(lib, 9, 1, 32, 8, 9, 8192)["join"] == ONE and plan(lib, 128, 1, 32, 8, 128, 8192)["join"] == ONE
    assert plan(lib, 129, 1, 32, 8, 129, 8192)["join"] == FOUR and plan(lib, 1 << 16, 1, 1024, 1, 1 << 16, 8192)["join"] == FOUR
