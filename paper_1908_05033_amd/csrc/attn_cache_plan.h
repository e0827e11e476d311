// Plan of a call of attention over a paged cache (host arithmetic).
#pragma once

struct AttnCachePlan {
    int slots, row_tiles;                    // chunks that all keys are cut into, at most that many and one more a sequence; tiles of 32 rows
};

// Two workgroups share a compute unit: 512 fill the card.
inline AttnCachePlan attn_cache_plan(int max_rows, int q_heads, int kv_heads)
{
    AttnCachePlan p;
    p.row_tiles = (int)(((long long)max_rows * (q_heads / kv_heads) + 31) / 32);
    const long long others = (long long)p.row_tiles * kv_heads;
    p.slots = others >= 512 ? 1 : (int)(512 / others);
    return p;
}
