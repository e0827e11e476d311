// Plan of the calls of attention over prompts (host arithmetic), and how packed sequences number their tiles (host and kernels).
#pragma once
#include <stdint.h>

// Heads of up to 64, 96 and 128 elements have kernels of their own.
constexpr int attn_width(int dim) { return dim <= 64 ? 64 : dim <= 96 ? 96 : 128; }

// Rows that a workgroup owns.  Few rows times heads: 32, and its waves split the keys; there 128 rows a workgroup leave compute units idle and
// make few long walks over the keys.  Forward, us, 128 rows / 32 rows a workgroup, rows x heads (causal):
//
//                   1024 x 8   2048 x 8   1024 x 32   2048 x 16   4096 x 8
//   bfloat16, 128   22 / 16    41 / 33    24 / 45     42 / 65     77 / 103
//   bfloat16, 64    19 / 11    34 / 19    19 / 19     34 / 25     62 / 40
//   binary32, 128   144 / 55   284 / 114  146 / 140   284 / 228   559 / 406
constexpr int64_t attn_fwd_few(int bytes, int width) { return bytes == 2 && width > 64 ? 32768 : 49152; }
constexpr int attn_fwd_rows(int bytes, int width, int rows, int heads) { return (int64_t)rows * heads < attn_fwd_few(bytes, width) ? 32 : 128; }

// The same for the queries' kernel of the backward pass (binary32: 64 rows).  Both kernels together, us, 128 (binary32: 64) rows / 32 rows
// a workgroup:
//
//                   1024 x 8    2048 x 8    1024 x 32   2048 x 16   4096 x 8
//   bfloat16, 128   63 / 57     97 / 93     76 / 111    107 / 147   186 / 236
//   bfloat16, 64    45 / 39     68 / 57     54 / 58     74 / 75     129 / 121
//   binary32, 128   183 / 145   397 / 338   335 / 391   599 / 669   1131 / 1225
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
