// Plan of a tiled product with group-scaled 4-bit weights: the tile's choice, and the packed channels that its waves read (host
// arithmetic; the kernel shares the latter).
#pragma once
#include "lm_kernels.h"

// The tile of 16 packed output channels that a lane reads whose wave begins at channel n0 (r: its place among the wave's 32).
// Channels are packed up to a multiple of 128 and the widest workgroups take 256: their waves past the packed channels
// read the last tile again, and store nothing.
__host__ __device__ inline int w4_channel_tile(int N, int n0, int r)
{
    const int tile = n0 / 16 + r / 16, last = dsq_w4_round(N) / 16 - 1;
    return tile < last ? tile : last;
}

struct W4Choice {
    int rows, channels, time;
};
// The choice with the least rounds of its workgroups over the 256 compute units times the time of a round.
template <int COUNT>
int w4_least_time(int M, int N, const W4Choice (&of)[COUNT])
{
    int best = 0;
    int64_t least = INT64_MAX;
    for (int i = 0; i < COUNT; ++i) {
        const int64_t count = (((int64_t)M + of[i].rows - 1) / of[i].rows) * (((int64_t)N + of[i].channels - 1) / of[i].channels);
        const int64_t time = (count + 255) / 256 * of[i].time;
        if (time < least) {
            least = time;
            best = i;
        }
    }
    return best;
}

// A large tile reads least and unpacks a code for most rows, a small one leaves no compute unit idle.  The times of a round are
// measured at K = 4096 and groups of 128, in microseconds with bfloat16 rows / 8-bit rows; another K and other groups are taken to scale
// all alike, which is not measured.  A round is one workgroup a compute unit, though two of the 8-bit 32x64 tile share one (its last
// lines below take less than rounds times time; larger tiles are ahead there).
//
//   rows x N        32x64      64x64      64x128     64x256     128x256
//   128 x 4096      14 / 9     20 / 12    25 / 17    37 / 26    63 / 40
//   256 x 4096      25 / 13    21 / 12    26 / 17    37 / 27    62 / 40
//   512 x 4096      48 / 23    41 / 23    30 / 18    39 / 27    63 / 41
//   1024 x 4096    103 / 47    80 / 46    59 / 37    47 / 32    67 / 42
//   2048 x 8192    388 / 185  325 / 200  225 / 146  179 / 121  158 / 101
constexpr W4Choice kW4Half[5] = {{32, 64, 13}, {64, 64, 20}, {64, 128, 27}, {64, 256, 41}, {128, 256, 76}};
constexpr W4Choice kW4Codes[5] = {{32, 64, 8}, {64, 64, 12}, {64, 128, 18}, {64, 256, 28}, {128, 256, 46}};

// Binary32 rows take three times the LDS and matrix instructions, and the kernel for a few rows is one of the choices:
//
//   rows x N       16x16 (w4_rows)   32x128   32x256   64x256
//   16 x 4096      12                29       45       77
//   64 x 4096      35                30       45       78
//   512 x 4096     236               71       61       83
//   1024 x 4096    468               139      112      101
constexpr W4Choice kW4Single[4] = {{16, 16, 9}, {32, 128, 33}, {32, 256, 58}, {64, 256, 100}};
