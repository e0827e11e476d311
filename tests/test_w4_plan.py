"""The plan of tiled products with 4-bit weights (CPU only: the planner's header in a small program): no wave reads channels
behind the packed ones, whatever tile is chosen."""
import os
import subprocess

import pytest

from paper_1908_05033_amd import binding as B

# One line "choice tile's rows tile's channels" out for each line "type M N" in (type 0: 16-bit rows, 1: 8-bit rows, 2: binary32
# ones); then, with every tile of the tables over many N, the number of lanes that read outside the packed channels, of lanes whose
# channel is not the one they read, and of waves that lie past the packed channels.
PROGRAM = r"""
#include <cstdio>
#include "w4_plan.h"
template <int COUNT>
void walk(const W4Choice (&of)[COUNT], int N, long &outside, long &other, long &past)
{
    for (int i = 0; i < COUNT; ++i)
        for (int n0 = 0; n0 < (N + of[i].channels - 1) / of[i].channels * of[i].channels; n0 += 32) {
            past += n0 >= dsq_w4_round(N);
            for (int r = 0; r < 32; ++r) {
                const int tile = w4_channel_tile(N, n0, r);
                outside += tile < 0 || 16 * tile + 16 > dsq_w4_round(N);
                other += n0 + r < N && tile != (n0 + r) / 16;
            }
        }
}
template <int COUNT>
void choose(const W4Choice (&of)[COUNT], int M, int N)
{
    const int i = w4_least_time(M, N, of);
    printf("%d %d %d\n", i, of[i].rows, of[i].channels);
}
int main()
{
    int type, M, N;
    while (scanf("%d %d %d", &type, &M, &N) == 3)
        type == 0 ? choose(kW4Half, M, N) : type == 1 ? choose(kW4Codes, M, N) : choose(kW4Single, M, N);
    long outside = 0, other = 0, past = 0;
    for (N = 1; N <= 1 << 24; N += N < 1200 ? 1 : N / 3 + 77) {
        walk(kW4Half, N, outside, other, past);
        walk(kW4Codes, N, outside, other, past);
        walk(kW4Single, N, outside, other, past);
    }
    printf("%ld %ld %ld\n", outside, other, past);
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("w4_plan")
    (d / "plan.cpp").write_text(PROGRAM)
    csrc = os.path.join(os.path.dirname(B.LIB_PATH), "csrc")
    cmd = ["g++", "-O2", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + csrc, str(d / "plan.cpp"), "-o", str(d / "plan")]
    proc = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert proc.returncode == 0, proc.stdout[-2000:]

    def run(cases):
        text = "".join("%d %d %d\n" % c for c in cases)
        out = subprocess.run([str(d / "plan")], input=text, stdout=subprocess.PIPE, text=True, check=True).stdout.split("\n")
        rows = [tuple(map(int, r.split())) for r in out if r]
        assert len(rows) == len(cases) + 1
        return rows[:-1], rows[-1]
    return run


def test_no_wave_reads_behind_the_packed_channels(plan):
    _, (outside, other, past) = plan([])
    assert past > 0                       # (there are waves without packed channels of their own)
    assert outside == 0 and other == 0


def test_wide_tiles_are_chosen_where_packed_channels_end_inside(plan):
    """The calls of test_gpu_w4_wide_tiles.py: 256 channels a workgroup, and an odd number of 128 packed ones."""
    from test_gpu_w4_wide_tiles import CASES
    chosen, _ = plan([c[:3] for c in CASES])
    for (_, _, N, rows), (_, tile_rows, channels) in zip(CASES, chosen):
        assert channels == 256 and tile_rows == rows and -(-N // 128) % 2 == 1
