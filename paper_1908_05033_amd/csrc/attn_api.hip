// C ABI of the calls between a block's products (see include/dsqconv.h): host-side validation and dispatch.
#include <math.h>

#include "../../include/dsqconv.h"
#include "attn_cache_plan.h"
#include "attn_kernels.h"
#include "dsq_kernels.h"

namespace {

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }
bool type_ok(dsq_dtype t) { return t == DSQ_F32 || t == DSQ_F16 || t == DSQ_BF16; }
const int kMaxRows = 1 << 21, kMaxHeads = 1024, kMaxSequences = 1 << 16, kMaxPage = 1 << 16, kMaxAxes = 16;
const int64_t kMaxKeys = 1LL << 30;          // of a sequence in a cache

dsq_status of_hip(hipError_t e) { return e == hipSuccess ? DSQ_OK : DSQ_ERR_HIP; }

// Distances of rows and heads: not negative, and a multiple of 16 bytes where there is more than one.
dsq_status distances_ok(int64_t row, int64_t head, int rows, int heads, dsq_dtype t)
{
    const int64_t unit = t == DSQ_F32 ? 4 : 8;
    if ((rows > 1 && row < 0) || (heads > 1 && head < 0)) return DSQ_ERR_SHAPE;
    if ((rows > 1 && row % unit) || (heads > 1 && head % unit)) return DSQ_ERR_ALIGN;
    return DSQ_OK;
}
// The same for an output, whose heads may not overlap.
dsq_status apart_ok(int64_t row, int64_t head, int rows, int heads, int dim, dsq_dtype t)
{
    const bool ok = rows <= 1 ? heads <= 1 || head >= dim
                    : heads <= 1 ? row >= dim
                    : head <= row ? head >= dim && row >= (heads - 1) * head + dim
                                  : row >= dim && head >= (rows - 1) * row + dim;
    return ok ? distances_ok(row, head, rows, heads, t) : DSQ_ERR_SHAPE;
}
int bits_of(int page)
{
    for (int b = 0; (1 << b) <= kMaxPage; ++b)
        if (page == 1 << b) return b;
    return -1;
}

size_t delta_bytes(int q_rows, int q_heads) { return ((size_t)q_rows * q_heads * 4 + 255) / 256 * 256; }

#define TRY(call)                                                                                                        \
    if (const dsq_status status_ = (call)) return status_

// What both passes of the norm and rotation have in common.
dsq_status heads_ok(dsq_dtype dtype, int rows, int q_heads, int kv_heads, int dim, const void *q, const void *k, const void *q_weight,
                    const void *k_weight, float eps, const int32_t *positions, int axes, const uint8_t *pair_axis, const float *frequencies,
                    int rope_dim)
{
    if (!type_ok(dtype)) return DSQ_ERR_UNSUPPORTED;
    if (rows < 0 || q_heads < 0 || kv_heads < 0 || q_heads + (int64_t)kv_heads == 0 || dim <= 0 || rope_dim < 0 || rope_dim > dim)
        return DSQ_ERR_SHAPE;
    if (rows > kMaxRows || q_heads > kMaxHeads || kv_heads > kMaxHeads || dim % 8 || dim > 256 || rope_dim % 16 || axes < 1 || axes > kMaxAxes)
        return DSQ_ERR_UNSUPPORTED;
    if (!(eps >= 0.0f && isfinite(eps))) return DSQ_ERR_RANGE;
    if (eps == 0.0f && (q_weight || k_weight)) return DSQ_ERR_UNSUPPORTED;
    if (rows == 0) return DSQ_OK;
    if ((q_heads && !q) || (kv_heads && !k) || (rope_dim && (!positions || !frequencies))) return DSQ_ERR_NULL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(q_weight) || !aligned16(k_weight) || !aligned16(positions) || !aligned16(pair_axis) ||
        !aligned16(frequencies))
        return DSQ_ERR_ALIGN;
    return DSQ_OK;
}

}  // namespace

extern "C" {

size_t dsq_qk_norm_rope_bwd_bytes(int rows, int q_heads, int kv_heads, int dim)
{
    if (rows <= 0 || rows > kMaxRows || q_heads < 0 || kv_heads < 0 || q_heads > kMaxHeads || kv_heads > kMaxHeads || q_heads + kv_heads == 0 ||
        dim <= 0 || dim % 8 || dim > 256)
        return 0;
    return (size_t)dsq_rope_bwd_parts(rows, q_heads, kv_heads, dim) * 2 * dim * 4;
}

size_t dsq_attention_bwd_bytes(int q_rows, int q_heads)
{
    if (q_rows <= 0 || q_rows > kMaxRows || q_heads <= 0 || q_heads > kMaxHeads) return 0;
    return delta_bytes(q_rows, q_heads) + dsq_attn_bwd_partial_bytes(q_rows, q_heads);
}

size_t dsq_attention_cache_bytes(int sequences, int max_rows, int q_heads, int kv_heads, int dim)
{
    if (sequences <= 0 || sequences > kMaxSequences || max_rows <= 0 || max_rows > kMaxRows || q_heads <= 0 || kv_heads <= 0 ||
        q_heads > kMaxHeads || kv_heads > kMaxHeads || q_heads % kv_heads || dim <= 0 || dim % 8 || dim > 128)
        return 0;
    return dsq_attn_cache_floats(sequences, max_rows, q_heads, kv_heads, dim) * 4;
}

dsq_status dsq_qk_norm_rope(const void *q, int64_t q_row, int64_t q_head, const void *k, int64_t k_row, int64_t k_head, const void *v,
                            int64_t v_row, int64_t v_head, dsq_dtype dtype, int rows, int q_heads, int kv_heads, int dim,
                            const void *q_weight, const void *k_weight, float eps, const int32_t *positions, int axes,
                            const uint8_t *pair_axis, const float *frequencies, int rope_dim, int interleaved, void *q_out,
                            int64_t q_out_row, int64_t q_out_head, void *k_out, int64_t k_out_row, int64_t k_out_head, void *k_cache,
                            void *v_cache, int64_t pages, int page, const int64_t *slots, void *hip_stream)
{
    TRY(heads_ok(dtype, rows, q_heads, kv_heads, dim, q, k, q_weight, k_weight, eps, positions, axes, pair_axis, frequencies, rope_dim));
    const bool cached = k_cache || v_cache || slots;
    if (rows == 0) return DSQ_OK;
    if ((q_heads && !q_out) || (kv_heads && !k_out && !cached) || (cached && (!k_cache || !v_cache || !slots || !v || !kv_heads))) return DSQ_ERR_NULL;
    if (!aligned16(v) || !aligned16(q_out) || !aligned16(k_out) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(slots))
        return DSQ_ERR_ALIGN;
    TRY(distances_ok(q_row, q_head, rows, q_heads, dtype));
    TRY(distances_ok(k_row, k_head, rows, kv_heads, dtype));
    if (cached) {
        TRY(distances_ok(v_row, v_head, rows, kv_heads, dtype));
        if (pages <= 0) return DSQ_ERR_SHAPE;
        if (pages > 0x7fffffff || bits_of(page) < 0) return DSQ_ERR_UNSUPPORTED;
    }
    if (q_heads) TRY(apart_ok(q_out_row, q_out_head, rows, q_heads, dim, dtype));
    if (k_out) TRY(apart_ok(k_out_row, k_out_head, rows, kv_heads, dim, dtype));
    // an output in the place of its input has to have its heads where the input has them
    if (q_heads && q_out == q && ((rows > 1 && q_out_row != q_row) || (q_heads > 1 && q_out_head != q_head))) return DSQ_ERR_UNSUPPORTED;
    if (k_out && k_out == k && ((rows > 1 && k_out_row != k_row) || (kv_heads > 1 && k_out_head != k_head))) return DSQ_ERR_UNSUPPORTED;
    DsqRopeArgs a;
    a.q = {q, q_row, q_head}; a.k = {k, k_row, k_head}; a.v = {v, v_row, v_head};
    a.q_out = {q_out, q_out_row, q_out_head}; a.k_out = {k_out, k_out_row, k_out_head};
    a.cache = {cached ? k_cache : nullptr, v_cache, pages, cached ? bits_of(page) : 0, slots};
    a.q_weight = q_weight; a.k_weight = k_weight; a.positions = positions; a.pair_axis = pair_axis; a.frequencies = frequencies;
    a.rows = rows; a.q_heads = q_heads; a.kv_heads = kv_heads; a.dim = dim; a.axes = axes; a.pairs = rope_dim / 2;
    a.interleaved = interleaved != 0; a.eps = eps;
    return of_hip(dsq_launch_qk_norm_rope(a, dtype, (hipStream_t)hip_stream));
}

dsq_status dsq_qk_norm_rope_bwd(const void *q, int64_t q_row, int64_t q_head, const void *k, int64_t k_row, int64_t k_head, dsq_dtype dtype,
                                int rows, int q_heads, int kv_heads, int dim, const void *q_weight, const void *k_weight, float eps,
                                const int32_t *positions, int axes, const uint8_t *pair_axis, const float *frequencies, int rope_dim,
                                int interleaved, const void *grad_q_out, int64_t grad_q_out_row, int64_t grad_q_out_head,
                                const void *grad_k_out, int64_t grad_k_out_row, int64_t grad_k_out_head, void *grad_q, int64_t grad_q_row,
                                int64_t grad_q_head, void *grad_k, int64_t grad_k_row, int64_t grad_k_head, float *grad_q_weight,
                                float *grad_k_weight, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    TRY(heads_ok(dtype, rows, q_heads, kv_heads, dim, q, k, q_weight, k_weight, eps, positions, axes, pair_axis, frequencies, rope_dim));
    if (eps == 0.0f && (grad_q_weight || grad_k_weight)) return DSQ_ERR_UNSUPPORTED;
    if (!aligned16(grad_q_weight) || !aligned16(grad_k_weight)) return DSQ_ERR_ALIGN;
    if (rows == 0) {
        for (float *w : {grad_q_weight, grad_k_weight})
            if (w) TRY(of_hip(dsq_launch_fill_zero((int32_t *)w, (size_t)dim, (hipStream_t)hip_stream)));
        return DSQ_OK;
    }
    if ((q_heads && (!grad_q_out || !grad_q)) || (kv_heads && (!grad_k_out || !grad_k)) || ((grad_q_weight || grad_k_weight) && !workspace))
        return DSQ_ERR_NULL;
    if (!aligned16(grad_q_out) || !aligned16(grad_k_out) || !aligned16(grad_q) || !aligned16(grad_k) || !aligned16(workspace)) return DSQ_ERR_ALIGN;
    TRY(distances_ok(q_row, q_head, rows, q_heads, dtype));
    TRY(distances_ok(k_row, k_head, rows, kv_heads, dtype));
    TRY(distances_ok(grad_q_out_row, grad_q_out_head, rows, q_heads, dtype));
    TRY(distances_ok(grad_k_out_row, grad_k_out_head, rows, kv_heads, dtype));
    if (q_heads) TRY(apart_ok(grad_q_row, grad_q_head, rows, q_heads, dim, dtype));
    if (kv_heads) TRY(apart_ok(grad_k_row, grad_k_head, rows, kv_heads, dim, dtype));
    if ((grad_q_weight || grad_k_weight) && workspace_bytes < dsq_qk_norm_rope_bwd_bytes(rows, q_heads, kv_heads, dim)) return DSQ_ERR_SIZE;
    const auto moved = [&](const void *o, int64_t row, int64_t head, const void *i, int64_t i_row, int64_t i_head, int heads) {
        return heads && o == i && ((rows > 1 && row != i_row) || (heads > 1 && head != i_head));
    };
    if (moved(grad_q, grad_q_row, grad_q_head, q, q_row, q_head, q_heads) || moved(grad_k, grad_k_row, grad_k_head, k, k_row, k_head, kv_heads) ||
        moved(grad_q, grad_q_row, grad_q_head, grad_q_out, grad_q_out_row, grad_q_out_head, q_heads) ||
        moved(grad_k, grad_k_row, grad_k_head, grad_k_out, grad_k_out_row, grad_k_out_head, kv_heads))
        return DSQ_ERR_UNSUPPORTED;
    DsqRopeBwdArgs a;
    a.q = {q, q_row, q_head}; a.k = {k, k_row, k_head};
    a.grad_q_out = {grad_q_out, grad_q_out_row, grad_q_out_head}; a.grad_k_out = {grad_k_out, grad_k_out_row, grad_k_out_head};
    a.grad_q = {grad_q, grad_q_row, grad_q_head}; a.grad_k = {grad_k, grad_k_row, grad_k_head};
    a.q_weight = q_weight; a.k_weight = k_weight; a.positions = positions; a.pair_axis = pair_axis; a.frequencies = frequencies;
    a.rows = rows; a.q_heads = q_heads; a.kv_heads = kv_heads; a.dim = dim; a.axes = axes; a.pairs = rope_dim / 2;
    a.interleaved = interleaved != 0; a.eps = eps;
    a.grad_q_weight = grad_q_weight; a.grad_k_weight = grad_k_weight; a.partial = (float *)workspace;
    return of_hip(dsq_launch_qk_norm_rope_bwd(a, dtype, (hipStream_t)hip_stream));
}

}  // extern "C"

namespace {

// A launch has fewer than 2^32 threads: tiles of 64 rows or more, and at most two more a sequence, of up to 512 threads.
bool tiles_fit(int rows, int heads, int sequences) { return (rows / 64 + 2LL * sequences) * heads <= 3 << 21; }

// What the calls of attention have in common.
dsq_status attention_ok(dsq_dtype dtype, int q_rows, int q_heads, int kv_heads, int dim, int sequences, float scale)
{
    if (!type_ok(dtype)) return DSQ_ERR_UNSUPPORTED;
    if (q_rows < 0 || q_heads <= 0 || kv_heads <= 0 || q_heads % kv_heads || dim <= 0 || sequences < 0) return DSQ_ERR_SHAPE;
    if (q_rows > kMaxRows || q_heads > kMaxHeads || dim % 8 || dim > 128 || sequences > kMaxSequences) return DSQ_ERR_UNSUPPORTED;
    if (!(scale > 0.0f && isfinite(scale))) return DSQ_ERR_RANGE;
    return DSQ_OK;
}
dsq_status prompts_ok(int q_rows, int k_rows, int q_heads, int kv_heads, int sequences, const int32_t *q_starts, const int32_t *k_starts)
{
    if (k_rows < 0 || (!q_starts && sequences != 1)) return DSQ_ERR_SHAPE;
    if (k_rows > kMaxRows || !tiles_fit(q_rows, q_heads, sequences) || !tiles_fit(k_rows, kv_heads, sequences)) return DSQ_ERR_UNSUPPORTED;
    if (!q_starts && k_starts) return DSQ_ERR_NULL;
    if (!aligned16(q_starts) || !aligned16(k_starts)) return DSQ_ERR_ALIGN;
    return DSQ_OK;
}

}  // namespace

extern "C" {

dsq_status dsq_attention(const void *q, int64_t q_row, int64_t q_head, const void *k, int64_t k_row, int64_t k_head, const void *v,
                         int64_t v_row, int64_t v_head, dsq_dtype dtype, int q_rows, int k_rows, int q_heads, int kv_heads, int dim,
                         const int32_t *q_starts, const int32_t *k_starts, int sequences, int causal, float scale, void *out,
                         int64_t out_row, int64_t out_head, float *lse, void *hip_stream)
{
    TRY(attention_ok(dtype, q_rows, q_heads, kv_heads, dim, sequences, scale));
    TRY(prompts_ok(q_rows, k_rows, q_heads, kv_heads, sequences, q_starts, k_starts));
    if (q_rows == 0 || sequences == 0) return DSQ_OK;
    if (!q || !out || (k_rows && (!k || !v))) return DSQ_ERR_NULL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(lse)) return DSQ_ERR_ALIGN;
    TRY(distances_ok(q_row, q_head, q_rows, q_heads, dtype));
    TRY(distances_ok(k_row, k_head, k_rows, kv_heads, dtype));
    TRY(distances_ok(v_row, v_head, k_rows, kv_heads, dtype));
    TRY(apart_ok(out_row, out_head, q_rows, q_heads, dim, dtype));
    DsqAttnArgs a;
    a.q = {q, q_row, q_head}; a.k = {k, k_row, k_head}; a.v = {v, v_row, v_head}; a.out = {out, out_row, out_head};
    a.lse = lse; a.q_starts = q_starts; a.k_starts = k_starts ? k_starts : q_starts;
    a.q_rows = q_rows; a.k_rows = k_rows; a.q_heads = q_heads; a.kv_heads = kv_heads; a.dim = dim;
    a.sequences = sequences; a.causal = causal != 0; a.scale = scale;
    return of_hip(dsq_launch_attention(a, dtype, (hipStream_t)hip_stream));
}

dsq_status dsq_attention_bwd(const void *q, int64_t q_row, int64_t q_head, const void *k, int64_t k_row, int64_t k_head, const void *v,
                             int64_t v_row, int64_t v_head, const void *out, int64_t out_row, int64_t out_head, const float *lse,
                             const void *grad_out, int64_t grad_out_row, int64_t grad_out_head, dsq_dtype dtype, int q_rows, int k_rows,
                             int q_heads, int kv_heads, int dim, const int32_t *q_starts, const int32_t *k_starts, int sequences, int causal,
                             float scale, void *grad_q, int64_t grad_q_row, int64_t grad_q_head, void *grad_k, int64_t grad_k_row,
                             int64_t grad_k_head, void *grad_v, int64_t grad_v_row, int64_t grad_v_head, void *workspace,
                             size_t workspace_bytes, void *hip_stream)
{
    TRY(attention_ok(dtype, q_rows, q_heads, kv_heads, dim, sequences, scale));
    TRY(prompts_ok(q_rows, k_rows, q_heads, kv_heads, sequences, q_starts, k_starts));
    if ((q_rows == 0 && k_rows == 0) || sequences == 0) return DSQ_OK;
    if ((q_rows && (!q || !out || !lse || !grad_out || !grad_q || !workspace)) || (k_rows && (!k || !v || !grad_k || !grad_v))) return DSQ_ERR_NULL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(lse) || !aligned16(grad_out) || !aligned16(grad_q) ||
        !aligned16(grad_k) || !aligned16(grad_v) || !aligned16(workspace))
        return DSQ_ERR_ALIGN;
    TRY(distances_ok(q_row, q_head, q_rows, q_heads, dtype));
    TRY(distances_ok(k_row, k_head, k_rows, kv_heads, dtype));
    TRY(distances_ok(v_row, v_head, k_rows, kv_heads, dtype));
    TRY(distances_ok(out_row, out_head, q_rows, q_heads, dtype));
    TRY(distances_ok(grad_out_row, grad_out_head, q_rows, q_heads, dtype));
    TRY(apart_ok(grad_q_row, grad_q_head, q_rows, q_heads, dim, dtype));
    TRY(apart_ok(grad_k_row, grad_k_head, k_rows, kv_heads, dim, dtype));
    TRY(apart_ok(grad_v_row, grad_v_head, k_rows, kv_heads, dim, dtype));
    if (workspace_bytes < dsq_attention_bwd_bytes(q_rows, q_heads)) return DSQ_ERR_SIZE;
    DsqAttnBwdArgs a;
    a.q = {q, q_row, q_head}; a.k = {k, k_row, k_head}; a.v = {v, v_row, v_head}; a.out = {out, out_row, out_head};
    a.grad_out = {grad_out, grad_out_row, grad_out_head}; a.grad_q = {grad_q, grad_q_row, grad_q_head};
    a.grad_k = {grad_k, grad_k_row, grad_k_head}; a.grad_v = {grad_v, grad_v_row, grad_v_head};
    a.lse = lse; a.delta = (float *)workspace;
    a.partial = (float *)((char *)workspace + (q_rows ? delta_bytes(q_rows, q_heads) : 0));
    a.partial_bytes = q_rows ? dsq_attn_bwd_partial_bytes(q_rows, q_heads) : 0;
    a.q_starts = q_starts; a.k_starts = k_starts ? k_starts : q_starts;
    a.q_rows = q_rows; a.k_rows = k_rows; a.q_heads = q_heads; a.kv_heads = kv_heads; a.dim = dim;
    a.sequences = sequences; a.causal = causal != 0; a.scale = scale;
    return of_hip(dsq_launch_attention_bwd(a, dtype, (hipStream_t)hip_stream));
}

dsq_status dsq_attention_cache(const void *q, int64_t q_row, int64_t q_head, dsq_dtype dtype, int rows, int q_heads, int kv_heads, int dim,
                               const int32_t *q_starts, int sequences, int max_rows, const void *k_cache, const void *v_cache, int64_t pages,
                               int page, const int32_t *page_table, int64_t table_row, int table_pages, const int32_t *lengths,
                               const uint64_t *tree, int tree_words, float scale, void *out, int64_t out_row, int64_t out_head,
                               void *workspace, size_t workspace_bytes, void *hip_stream)
{
    TRY(attention_ok(dtype, rows, q_heads, kv_heads, dim, sequences, scale));
    const int bits = bits_of(page);
    if (max_rows <= 0 || pages < 0 || table_pages < 0 || (!q_starts && rows != sequences) || (tree && tree_words <= 0)) return DSQ_ERR_SHAPE;
    if (max_rows > kMaxRows || pages > 0x7fffffff || bits < 0 || (int64_t)table_pages << bits > kMaxKeys) return DSQ_ERR_UNSUPPORTED;
    if (rows == 0 || sequences == 0) return DSQ_OK;
    const AttnCachePlan p = attn_cache_plan(max_rows, q_heads, kv_heads, sequences, (int64_t)table_pages << bits);
    // (a launch has fewer than 2^32 threads: 512 a chunk, 64 a row and head or four)
    if ((int64_t)sequences * p.row_tiles * kv_heads >= 1 << 22 || (int64_t)rows * q_heads >= 1 << 26 ||
        (((int64_t)table_pages << bits) / 128 + 1) * sequences > 1 << 30 || (int64_t)max_rows * (q_heads / kv_heads) > 1 << 30)
        return DSQ_ERR_UNSUPPORTED;
    if (!q || !out || !lengths || !workspace || (pages && (!k_cache || !v_cache)) || (table_pages && !page_table)) return DSQ_ERR_NULL;
    if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(q_starts) || !aligned16(page_table) || !aligned16(lengths) ||
        !aligned16(tree) || !aligned16(out) || !aligned16(workspace))
        return DSQ_ERR_ALIGN;
    if (sequences > 1 && table_row < 0) return DSQ_ERR_SHAPE;
    TRY(distances_ok(q_row, q_head, rows, q_heads, dtype));
    TRY(apart_ok(out_row, out_head, rows, q_heads, dim, dtype));
    if (workspace_bytes < dsq_attention_cache_bytes(sequences, max_rows, q_heads, kv_heads, dim)) return DSQ_ERR_SIZE;
    DsqAttnCacheArgs a;
    a.q = {q, q_row, q_head}; a.out = {out, out_row, out_head}; a.k_cache = k_cache; a.v_cache = v_cache; a.q_starts = q_starts;
    a.table = page_table; a.lengths = lengths; a.tree = tree; a.pages = pages; a.table_row = table_row;
    a.rows = rows; a.q_heads = q_heads; a.kv_heads = kv_heads; a.dim = dim; a.sequences = sequences; a.max_rows = max_rows;
    a.page_bits = bits; a.table_pages = table_pages; a.tree_words = tree_words; a.scale = scale; a.partial = (float *)workspace;
    return of_hip(dsq_launch_attention_cache(a, dtype, (hipStream_t)hip_stream));
}

}  // extern "C"
