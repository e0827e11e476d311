// Plan of a call of attention over a paged cache (host arithmetic), and how the keys of its sequences are cut into chunks (host and kernels).
#pragma once
#include <stdint.h>

constexpr int kAttnUnit = 128;               // keys a chunk is a multiple of: a block of 32 for each of four waves

// Chunks have the same number of units for all sequences: what all have together over the slots, one at least.  They are numbered as
// tiles of sequences are: sequence s has them from (units before it) / units a chunk + s on.  All numbers are below slots + sequences.
constexpr int attn_units(int length) { return (length + kAttnUnit - 1) / kAttnUnit; }
constexpr int attn_chunk_units(int total, int slots) { return total > slots ? (total + slots - 1) / slots : 1; }
constexpr int attn_first_chunk(int before, int units, int s) { return before / units + s; }
// Keys of a chunk of so many units: a sequence has at most 2^30.
constexpr int attn_chunk_keys(int units) { return (units < 1 << 23 ? units : 1 << 23) * kAttnUnit; }

struct AttnCachePlan {
    bool tiles;                              // more than 32 rows a key head: four waves share tiles of keys
    bool single;                             // every sequence is one chunk: nothing to join
    int row_tiles, slots;                    // tiles of rows; chunks that all keys are cut into (and one more a sequence); 0: single
};

// `keys`: the most that a sequence can have.
inline AttnCachePlan attn_cache_plan(int max_rows, int q_heads, int kv_heads, int sequences, int64_t keys)
{
    AttnCachePlan p;
    const int64_t rows = (int64_t)max_rows * (q_heads / kv_heads);
    p.tiles = rows > 32;
    p.row_tiles = p.tiles ? (int)((rows + 127) / 128) : 1;
    const int64_t others = (int64_t)p.row_tiles * kv_heads;
    // Two workgroups share a compute unit.  512 chunks fill the card, and one sequence's are alike; those of several end where their
    // sequences do, and twice as many even that out (32 of up to 8192 keys 104 us for 119; one of 131072: 57 for 54, its join 10 for 8).
    const int64_t most = p.tiles || sequences == 1 ? 512 : 1024;
    p.slots = others >= most ? 1 : (int)(most / others);
    p.single = !p.tiles && keys <= 1024;
    if (p.single) p.slots = 0;
    return p;
}

// The kernel that joins chunks.  Many chunks a row: a workgroup of 16 waves for each; else a wave for a row, or for four heads of it where there are many.
enum AttnCacheJoin { kJoinNone, kJoinSixteen, kJoinOne, kJoinFour };
inline AttnCacheJoin attn_cache_join(const AttnCachePlan &p, int rows, int q_heads, int sequences)
{
    const int64_t all = (int64_t)rows * q_heads;
    return p.single ? kJoinNone : p.slots / sequences >= 16 && all <= 1024 ? kJoinSixteen : all <= 4096 ? kJoinOne : kJoinFour;
}
