"""Rules and numbers of the kernels for prompts, compiled from the header that the library uses: which kernel a call takes, and that tiles of packed
sequences neither meet nor go missing."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import test_gpu_attention_many_rows as many

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
SOURCE = """#include "%s/paper_1908_05033_amd/csrc/attn_prompt_plan.h"
extern "C" {
int width(int dim) { return attn_width(dim); }
int fwd_rows(int bytes, int width, int rows, int heads) { return attn_fwd_rows(bytes, width, rows, heads); }
int bwd_rows(int bytes, int width, int rows, int heads) { return attn_bwd_rows(bytes, width, rows, heads); }
int first_tile(int start, int tile, int s) { return attn_first_tile(start, tile, s); }
int tiles(int rows, int tile, int sequences, int packed) { return attn_tiles(rows, tile, sequences, packed); }
int turns(int tiles, int sequences) { return attn_turns(tiles, sequences); }
int tile_of_turn(int turn, int tiles, int sequences) { return attn_tile_of_turn(turn, tiles, sequences); }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SOURCE % ROOT)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", str(d / "plan.so"), str(d / "plan.cpp")], check=True)
    return ctypes.CDLL(str(d / "plan.so"))


def test_rule(plan):
    assert [plan.width(d) for d in (8, 64, 72, 96, 104, 128)] == [64, 64, 96, 96, 128, 128]
    for bytes_, width, fwd, bwd in ((2, 64, 49152, 49152), (2, 96, 32768, 32768), (2, 128, 32768, 32768), (4, 64, 49152, 32768), (4, 96, 49152, 32768),
                                    (4, 128, 49152, 32768)):
        many_rows = 64 if bytes_ == 4 else 128
        assert plan.fwd_rows(bytes_, width, fwd // 8 - 1, 8) == 32 and plan.fwd_rows(bytes_, width, fwd // 8, 8) == 128
        assert plan.bwd_rows(bytes_, width, bwd // 8 - 1, 8) == 32 and plan.bwd_rows(bytes_, width, bwd // 8, 8) == many_rows
        # (rows times heads pass 2^31)
        assert plan.fwd_rows(bytes_, width, 1 << 21, 1024) == 128 and plan.bwd_rows(bytes_, width, 1 << 21, 1024) == many_rows


@pytest.mark.parametrize("dtype", BYTES)
def test_shapes_of_many_rows_take_their_kernels(plan, dtype):
    """All types and widths, forward and backward; the kernels of few rows have tests of their own."""
    b = BYTES[dtype]
    assert {plan.width(d) for d in many.DIMS} == {64, 96, 128}
    for name, (q_sizes, _, hq, _, first) in many.SHAPES.items():
        rows = sum(q_sizes) + 2 * first
        for d in many.DIMS:
            assert plan.fwd_rows(b, plan.width(d), rows, hq) == 128 and plan.bwd_rows(b, plan.width(d), rows, hq) == (64 if b == 4 else 128), (name, d)
    # the other tests there: rows x heads
    for rows in (1024, 1030, 1040, 1050, 1100):
        for w in (64, 96, 128):
            assert plan.fwd_rows(b, w, rows, 48) == 128 and plan.bwd_rows(b, w, rows, 48) > 32
    for w in (64, 96, 128):
        kinds = {(plan.fwd_rows(b, w, rows, 48), plan.bwd_rows(b, w, rows, 48) > 32) for rows in (682, 683, 1023, 1024)}
        assert {k[0] for k in kinds} == {32, 128} and {k[1] for k in kinds} == {False, True}


def sequences_of(rs):
    n = rs.randint(1, 60)
    return np.concatenate([[0], np.cumsum(rs.randint(0, 2, n) * (10 ** rs.uniform(0, 3, n)).astype(int))]) + rs.randint(0, 200)


@pytest.mark.parametrize("tile", [32, 64, 128])
def test_numbers_of_tiles(plan, tile):
    """Every row of every sequence is in one tile, tiles of two sequences do not meet, and all numbers are below the launch's."""
    rs = np.random.RandomState(tile)
    for _ in range(200):
        starts = sequences_of(rs)
        n, rows = len(starts) - 1, int(starts[-1]) + rs.randint(0, 3) * rs.randint(0, 100)
        total = plan.tiles(rows, tile, n, 1)
        first = [plan.first_tile(int(s), tile, i) for i, s in enumerate(starts)]
        need = [-(-int(b - a) // tile) for a, b in zip(starts, starts[1:])]
        assert all(f + m <= g for f, m, g in zip(first, need, first[1:])) and first[-2] + need[-1] <= total
    assert [plan.tiles(r, tile, 1, 0) for r in (1, tile, tile + 1)] == [1, 1, 2]


def test_turns_take_every_tile_once(plan):
    for tiles, n in ((1, 1), (7, 1), (17, 4), (5, 9), (64, 16), (1000, 37), (70, 70)):
        turns = plan.turns(tiles, n)
        at = [plan.tile_of_turn(i, tiles, n) for i in range(turns)]
        assert sorted(t for t in at if t >= 0) == list(range(tiles)) and max(at) < tiles and len([t for t in at if t < 0]) == turns - tiles
    # one sequence: from the last tile to the first
    assert [plan.tile_of_turn(i, 4, 1) for i in range(4)] == [3, 2, 1, 0]
