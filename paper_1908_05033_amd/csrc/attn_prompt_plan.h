// Plan of the calls of attention over prompts (host arithmetic), and how packed sequences number their tiles (host and kernels).
#pragma once
#include <stdint.h>

// Heads of up to 64, 96 and 128 elements have kernels of their own.
constexpr int attn_width(int dim) { return dim <= 64 ? 64 : dim <= 96 ? 96 : 128; }

// Rows that a workgroup owns.  Few rows times heads: 32, and its waves split the keys; there 128 rows a workgroup leave compute units idle and
// make few long walks over the keys.  Forward, us, 128 rows / 32 rows a workgroup, rows x heads (causal; float16 as bfloat16 within 6 %):
//
//                   1024 x 8   2048 x 8   1024 x 32   2048 x 16   4096 x 8    1536 x 32   6144 x 8
//   bfloat16, 64    19 / 11    34 / 19    19 / 18     34 / 25     63 / 39     27 / 31     94 / 79
//   bfloat16, 96    20 / 14    37 / 29    24 / 38     40 / 56     84 / 95     37 / 72     129 / 214
//   bfloat16, 128   22 / 16    40 / 32    24 / 43     43 / 62     78 / 100    40 / 79     140 / 209
//   binary32, 64    76 / 28    150 / 59   78 / 71     151 / 115   297 / 206   141 / 140   549 / 444
//   binary32, 96    113 / 42   225 / 88   116 / 107   226 / 176   445 / 312   172 / 212   669 / 680
//   binary32, 128   142 / 55   283 / 115  146 / 140   283 / 230   561 / 412   217 / 276   842 / 891
//
// (The product alone is not all: at 64 elements 6144 rows of 8 heads would take a sixth to a fifth less with 32 rows a workgroup.)
constexpr int64_t attn_fwd_few(int bytes, int width) { return bytes == 2 && width > 64 ? 32768 : 49152; }
constexpr int attn_fwd_rows(int bytes, int width, int rows, int heads) { return (int64_t)rows * heads < attn_fwd_few(bytes, width) ? 32 : 128; }

// The same for the queries' kernel of the backward pass (binary32: 64 rows).  Both kernels together, us, 128 (binary32: 64) rows / 32 rows
// a workgroup:
//
//                   1024 x 8    2048 x 8    1024 x 32   2048 x 16   4096 x 8      1536 x 32   6144 x 8
//   bfloat16, 64    45 / 39     67 / 57     53 / 58     74 / 74     128 / 120     81 / 93     244 / 248
//   bfloat16, 96    53 / 50     81 / 83     65 / 98     91 / 130    156 / 211     100 / 167   295 / 447
//   bfloat16, 128   63 / 56     96 / 93     75 / 111    106 / 147   183 / 235     117 / 190   348 / 496
//   binary32, 64    101 / 79    218 / 183   200 / 214   363 / 365   686 / 664     385 / 436   1330 / 1443
//   binary32, 96    149 / 120   321 / 277   273 / 323   484 / 551   913 / 1008    589 / 659   2067 / 2194
//   binary32, 128   182 / 145   397 / 340   335 / 394   600 / 673   1135 / 1231   721 / 804   2566 / 2681
//
// (Here 1024 rows of 32 heads of 64 elements, bfloat16, would take a twelfth less with 128.)
constexpr int64_t attn_bwd_few(int bytes, int width) { return bytes == 2 && width == 64 ? 49152 : 32768; }
constexpr int attn_bwd_rows(int bytes, int width, int rows, int heads)
{
    return (int64_t)rows * heads < attn_bwd_few(bytes, width) ? 32 : bytes == 4 ? 64 : 128;
}

// Tiles of `tile` rows: sequence s has its own from number starts[s] / tile + s on, which leaves room for as many as it
// needs without a sum over the sequences before it; tiles past its end have nothing to do.
constexpr int attn_first_tile(int start, int tile, int s) { return start / tile + s; }
constexpr int attn_tiles(int rows, int tile, int sequences, bool packed) { return packed ? rows / tile + sequences : (rows + tile - 1) / tile; }

// Order of the tiles: their numbers in as many bands as there are sequences, from the end of each band to its start, the bands in turn.  In sequences of
// one length (or one sequence) those are the sequences' tiles, and the last ones, the longest of a causal prompt, go first.
constexpr int attn_turns(int tiles, int sequences) { return (tiles + sequences - 1) / sequences * sequences; }
constexpr int attn_tile_of_turn(int turn, int tiles, int sequences)
{
    return tiles - 1 - turn % sequences * ((tiles + sequences - 1) / sequences) - turn / sequences;      // (negative: none)
}
