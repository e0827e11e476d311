// Internal launch interface of the attention calls (attn_api.hip): norms and rotation of heads, attention over prompts and over a
// paged cache.  Arguments have already been validated by the caller.
#pragma once
#include "lm_kernels.h"

// Heads in memory: [rows][heads][dim], the elements of a head side by side; distances in elements.
struct DsqHeads {
    const void *p;
    int64_t row, head;
};
struct DsqHeadsOut {
    void *p;
    int64_t row, head;
};

// A paged cache: [pages][kv heads][page][dim] each; k may be null where there is none.
struct DsqCacheOut {
    void *k, *v;
    int64_t pages;
    int page_bits;
    const int64_t *slots;                    // of each row: page * page size + place; others than 0 .. slots - 1 are not written
};

struct DsqRopeArgs {
    DsqHeads q, k, v;                        // v: null without a cache
    DsqHeadsOut q_out, k_out;                // k_out may be null with a cache
    DsqCacheOut cache;
    const void *q_weight, *k_weight;         // null: ones
    const int32_t *positions;                // [axes][rows]
    const uint8_t *pair_axis;                // [pairs] or null: axis 0
    const float *frequencies;                // [pairs]
    int rows, q_heads, kv_heads, dim, axes, pairs, interleaved;
    float eps;                               // 0: no norm
};
hipError_t dsq_launch_qk_norm_rope(const DsqRopeArgs &a, int type, hipStream_t stream);

struct DsqRopeBwdArgs {
    DsqHeads q, k, grad_q_out, grad_k_out;
    DsqHeadsOut grad_q, grad_k;
    const void *q_weight, *k_weight;
    const int32_t *positions;
    const uint8_t *pair_axis;
    const float *frequencies;
    int rows, q_heads, kv_heads, dim, axes, pairs, interleaved;
    float eps;
    float *grad_q_weight, *grad_k_weight;    // may be null
    float *partial;                          // [dsq_rope_bwd_parts][2][dim], unused without gradients of weights
};
int dsq_rope_bwd_parts(int rows, int q_heads, int kv_heads, int dim);
hipError_t dsq_launch_qk_norm_rope_bwd(const DsqRopeBwdArgs &a, int type, hipStream_t stream);

struct DsqAttnArgs {
    DsqHeads q, k, v;
    DsqHeadsOut out;
    float *lse;                              // [q_heads][q_rows] or null
    const int32_t *q_starts, *k_starts;      // [sequences + 1]; null: one sequence of all rows
    int q_rows, k_rows, q_heads, kv_heads, dim, sequences, causal;
    float scale;
};
hipError_t dsq_launch_attention(const DsqAttnArgs &a, int type, hipStream_t stream);

struct DsqAttnBwdArgs {
    DsqHeads q, k, v, out, grad_out;
    DsqHeadsOut grad_q, grad_k, grad_v;
    const float *lse;
    float *delta;                            // [q_heads][q_rows]: sums of out * grad_out
    float *partial;                          // room for sums of dk and dv of parts of the rows
    size_t partial_bytes;
    const int32_t *q_starts, *k_starts;
    int q_rows, k_rows, q_heads, kv_heads, dim, sequences, causal;
    float scale;
};
// Room that joins sums over parts of the rows where there are few keys.
size_t dsq_attn_bwd_partial_bytes(int q_rows, int q_heads);
hipError_t dsq_launch_attention_bwd(const DsqAttnBwdArgs &a, int type, hipStream_t stream);

struct DsqAttnCacheArgs {
    DsqHeads q;
    DsqHeadsOut out;
    const void *k_cache, *v_cache;           // [pages][kv_heads][page][dim]
    const int32_t *q_starts;                 // [sequences + 1]; null: a row each
    const int32_t *table;                    // [sequences] rows of table_row
    const int32_t *lengths;                  // [sequences]
    const uint64_t *tree;                    // [rows][tree_words] or null: a chain
    int64_t pages, table_row;
    int rows, q_heads, kv_heads, dim, sequences, max_rows, page_bits, table_pages, tree_words;
    float scale;
    float *partial;
};
size_t dsq_attn_cache_floats(int sequences, int max_rows, int q_heads, int kv_heads, int dim);
hipError_t dsq_launch_attention_cache(const DsqAttnCacheArgs &a, int type, hipStream_t stream);
