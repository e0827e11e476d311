// Plan of a call of attention over a paged cache (host arithmetic).
#pragma once
#include <stdint.h>

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
