// Attention of single tokens, and of trees of drafted tokens, over a paged cache.
//
// The rows of a key head are the drafted tokens of a sequence times the query heads that share it; 32 of them are one tile.  A
// sequence's keys are cut into chunks of one length for all sequences, so that a batch of many lengths fills the card evenly, and a
// workgroup takes a chunk of a key head for a tile of rows: its four waves take blocks of 32 keys in turn, each with the running
// maximum and sum of a softmax, and join in LDS.  A sequence of one chunk is finished there; the others leave normed rows
// and the logarithms of their sums, which a second kernel joins.  Keys and values are read once for 32 rows, in whole rows of a page,
// and go through LDS of the wave's own, so a wave waits for nothing but its own loads.
#include "attn_cache_plan.h"
#include "attn_device.h"

namespace {

constexpr int kUnit = 128;                   // keys a chunk is a multiple of: a block for each wave

struct Chunk {
    int sequence, first, count, chunks;      // first: key; count: keys; chunks: of the sequence (0 without keys)
    int length;
};

__device__ __forceinline__ int sum_to(int v, int lane)
{
    for (int off = 1; off < 64; off <<= 1) {
        const int u = __shfl_up(v, off);
        if (lane >= off) v += u;
    }
    return v;
}

__device__ __forceinline__ int length_of(const DsqAttnCacheArgs &a, int s) { return clamped(a.lengths[s], a.table_pages << a.page_bits); }

// Units of keys a chunk has: the same for all sequences.
__device__ __forceinline__ int chunk_units(const DsqAttnCacheArgs &a, int slots, int lane)
{
    int total = 0;
    for (int s = lane; s < a.sequences; s += 64) total += (length_of(a, s) + kUnit - 1) / kUnit;
    for (int off = 32; off > 0; off >>= 1) total += __shfl_xor(total, off);
    const int c = (total + slots - 1) / slots;
    return c > 0 ? c : 1;
}

// Chunks are numbered as tiles of sequences are: sequence s has them from (units before it) / units a chunk + s on.  Either the chunk of
// a number, or (`number` negative) the first number of sequence `s`; all 64 lanes take part.
__device__ __forceinline__ int first_chunk(const DsqAttnCacheArgs &a, int units, int number, int &s)
{
    const int lane = threadIdx.x & 63;
    int before = 0, found = -1, at = -1;
    for (int base = 0; base < a.sequences; base += 64) {
        const int i = base + lane, mine = i < a.sequences ? (length_of(a, i) + kUnit - 1) / kUnit : 0;
        const int sum = sum_to(mine, lane), slot = (before + sum - mine) / units + i;
        const uint64_t ok = __ballot(i < a.sequences && (number < 0 ? i <= s : slot <= number));
        if (ok == 0) break;
        const int last = 63 - __clzll((long long)ok);
        found = base + last;
        at = __shfl(slot, last);
        before += __shfl(sum, 63);
        if (last < 63) break;
    }
    s = __builtin_amdgcn_readfirstlane(found);
    return __builtin_amdgcn_readfirstlane(at);
}

// Where key j of a sequence lies: a row of [pages][kv heads][page], negative where there is none.
struct Pages {
    const int32_t *table;
    int64_t pages;
    int table_pages, bits, kv, kv_heads, length;
    __device__ __forceinline__ int64_t row(int j) const
    {
        if (j >= length) return -1;
        const int p = j >> bits;
        const int id = p < table_pages ? table[p] : -1;
        if (id < 0 || id >= pages) return -1;
        return ((((int64_t)id * kv_heads + kv) << bits) + (j & ((1 << bits) - 1)));
    }
};

// Which of the 32 keys from j0 on a drafted token sees: those before the drafted ones (from `context` on), and of these the ones in its mask.
struct Tree {
    const uint64_t *words;                   // of the token, or null: the drafted tokens up to `token`
    int count, token, context;
    __device__ __forceinline__ uint64_t word(int i) const { return i < count ? words[i] : 0; }
    __device__ __forceinline__ uint32_t mask(int j0) const
    {
        const int b = j0 - context;
        if (b <= -32) return 0xffffffffu;
        if (!words) {
            const int n = token - b + 1;
            return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1;
        }
        if (b < 0) return (uint32_t)(word(0) << -b) | ((1u << -b) - 1);
        const int w = b / 64, at = b % 64;
        uint64_t bits = word(w) >> at;
        if (at > 32) bits |= word(w + 1) << (64 - at);
        return (uint32_t)bits;
    }
};

template <class E>
struct CacheKeys {
    const E *k, *v;
    Pages pages;
    Tree tree;
    int first, n, dim;
    __device__ int count() const { return n; }
    __device__ bool seen(int j) const { return pages.row(first + j) >= 0 && (tree.mask(first + j) & 1); }
    __device__ const E *key(int j) const { return k + pages.row(first + j) * dim; }
    __device__ const E *value(int j) const { return v + pages.row(first + j) * dim; }
};

template <class E, int HD>
__global__ __launch_bounds__(256, sizeof(E) == 2 ? 2 : 1) void attn_cache_kernel(DsqAttnCacheArgs a, int slots, int row_tiles)
{
    typedef Tile<E, HD> T;
    typedef typename Operand<E>::type V8;
    constexpr int STEPS = HD / 16, DT = HD / 32, PIECES = 32 * T::UNITS / 64, PITCH = 33;
    constexpr int WAVE_BYTES = HD * PITCH * 4 > 64 * HD * (int)sizeof(E) ? HD * PITCH * 4 : 64 * HD * (int)sizeof(E);
    __shared__ __align__(16) char room[4 * WAVE_BYTES];
    __shared__ float stat[4][2][32];
    __shared__ uint32_t seen_by[4][32];

    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), r = lane & 31, h = lane >> 5;
    const int per = row_tiles * a.kv_heads, number = blockIdx.x / per;
    const int kv = blockIdx.x % per % a.kv_heads, rt = blockIdx.x % per / a.kv_heads;
    const int group = a.q_heads / a.kv_heads, most_rows = a.max_rows * group;

    const int units = chunk_units(a, slots, lane);
    int s;
    const int slot0 = first_chunk(a, units, number, s);
    if (s < 0) return;
    const int length = length_of(a, s), chunk = units * kUnit;
    if ((int64_t)(number - slot0) * chunk >= length && number != slot0) return;
    const int first = (number - slot0) * chunk, end = length - first < chunk ? length : first + chunk;
    const bool whole = length <= chunk;
    const int t0 = a.q_starts ? clamped(a.q_starts[s], a.rows) : s;
    const int tokens = a.q_starts ? clamped(a.q_starts[s + 1], a.rows) - t0 : 1;
    const int mine = tokens < a.max_rows ? tokens : a.max_rows;
    if (rt * 32 >= mine * group) return;

    const int row = rt * 32 + r, token = row / group, head = kv * group + row % group;
    const bool there = token < mine;
    const Pages pages = {a.table + s * a.table_row, a.pages, a.table_pages, a.page_bits, kv, a.kv_heads, length};
    const Tree tree = {a.tree && there ? a.tree + (int64_t)(t0 + token) * a.tree_words : nullptr, a.tree_words, token, length - tokens};
    const E *kp = (const E *)a.k_cache, *vp = (const E *)a.v_cache;

    V8 q[STEPS];
    {
        const E *qp = (const E *)a.q.p + (int64_t)(t0 + token) * a.q.row + head * a.q.head;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) q[i] = load_unit8(qp, 2 * i + h, a.dim, there);
    }

    E *ks = reinterpret_cast<E *>(room + wave * WAVE_BYTES), *vs = ks + 32 * HD;
    v4u kr[PIECES], vr[PIECES];
    uint32_t valid;                          // of the 32 keys under way
    auto fetch = [&](int64_t place) {        // place: of key lane % 32 of the block
        valid = (uint32_t)__ballot(place >= 0 && lane < 32);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int piece = lane + 64 * i, u = piece % T::UNITS;
            const int64_t at = __shfl(place, piece / T::UNITS);
            const bool ok = at >= 0 && u * T::PER < a.dim;
            kr[i] = ok ? *reinterpret_cast<const v4u *>(kp + at * a.dim + u * T::PER) : v4u{0, 0, 0, 0};
            vr[i] = ok ? *reinterpret_cast<const v4u *>(vp + at * a.dim + u * T::PER) : v4u{0, 0, 0, 0};
        }
    };

    const float c = a.scale * kLog2e;
    float m = kNoKey, l = 0.0f;
    uint32_t any = 0;
    v16f o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;

    int j = first + wave * 32;
    int64_t next = j < end ? pages.row(j + r) : -1;
    if (j < end) fetch(next);
    next = j + 128 < end ? pages.row(j + 128 + r) : -1;
    for (; j < end; j += 128) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int piece = lane + 64 * i, at = T::place(piece / T::UNITS, piece % T::UNITS);
            *reinterpret_cast<v4u *>(ks + at) = kr[i];
            *reinterpret_cast<v4u *>(vs + at) = vr[i];
        }
        wave_order();
        uint32_t mask = valid & (there ? tree.mask(j) : 0);
        if (j + 128 < end) {
            fetch(next);
            next = j + 256 < end ? pages.row(j + 256 + r) : -1;
        }
        any |= mask;
        v16f x;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.0f;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) x = multiply(T::row_operand(ks, r, i, h), q[i], x);
        if (__any(mask != 0xffffffffu)) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = mask >> (8 * (i / 4) + 4 * h + i % 4) & 1 ? x[i] : -INFINITY;
        }
        float most = x[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) most = __builtin_elementwise_maximum(most, x[i]);
        most = both_max(most) * c;
        if (__any(most > m + 8.0f)) {
            const float raised = most > m ? most : m, f = __builtin_amdgcn_exp2f(m - raised);
            m = raised;
            l *= f;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= f;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], c, -m));
            l += x[i];
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const V8 p = operand_of<E>(x, half);
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] = multiply(T::column_operand(vs, half * 16, d * 32, lane), p, o[d]);
        }
        wave_order();
    }

    // ---- the four waves' rows: [HD][PITCH] of each in the room of its tiles
    float *mine_o = reinterpret_cast<float *>(room + wave * WAVE_BYTES);
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) mine_o[(d * 32 + 8 * (i / 4) + 4 * h + i % 4) * PITCH + r] = o[d][i];
    l = both_sum(l);
    if (h == 0) {
        stat[wave][0][r] = m;
        stat[wave][1][r] = l;
        seen_by[wave][r] = any;
    }
    __syncthreads();
    const int64_t place = ((int64_t)number * a.kv_heads + kv) * most_rows;
    float *rows_out = a.partial, *logs = a.partial + (int64_t)(slots + a.sequences) * a.kv_heads * most_rows * a.dim;
    const int live = mine * group - rt * 32;
    for (int i = wave; i < 32 && i < live; i += 4) {
        float top = kNoKey;
        uint32_t seen = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = __builtin_elementwise_maximum(top, stat[w][0][i]), seen |= seen_by[w][i];
        float f[4], sum = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            f[w] = __builtin_amdgcn_exp2f(stat[w][0][i] - top);
            sum = __builtin_fmaf(stat[w][1][i], f[w], sum);
        }
        const int of = rt * 32 + i;
        float y[2];
        bool bad = false;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int d = lane + 64 * e;
            y[e] = 0.0f;
            if (d < HD) {
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    y[e] = __builtin_fmaf(reinterpret_cast<const float *>(room + w * WAVE_BYTES)[d * PITCH + i], f[w], y[e]);
                y[e] = seen ? y[e] / sum : 0.0f;
            }
            bad |= !is_finite(y[e]);
        }
        float log2 = top + __builtin_amdgcn_logf(sum);
        if (__any(bad)) {
            const int tk = of / group;
            const Tree its = {a.tree ? a.tree + (int64_t)(t0 + tk) * a.tree_words : nullptr, a.tree_words, tk, length - tokens};
            const CacheKeys<E> keys = {kp, vp, pages, its, first, end - first, a.dim};
            log2 = row_again<E>((const E *)a.q.p + (int64_t)(t0 + tk) * a.q.row + (kv * group + of % group) * a.q.head, a.dim, c, keys, y);
        }
        // (a row whose scores are all -inf is NaN by the formula, but only where no other chunk has more)
        if (!(log2 > kNoKey) && log2 == log2) log2 = kNoKey;
        if (whole) {
            E *to = (E *)a.out.p + (int64_t)(t0 + of / group) * a.out.row + (kv * group + of % group) * a.out.head;
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (lane + 64 * e < a.dim) to[lane + 64 * e] = (E)y[e];
        } else {
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (lane + 64 * e < a.dim) rows_out[(place + of) * a.dim + lane + 64 * e] = y[e];
            if (lane == 0) logs[place + of] = seen ? log2 : -INFINITY;
        }
    }
}

// The chunks of a row, weighted by their sums: one workgroup a row of a head, its waves take chunks in turn.
template <class E>
__global__ __launch_bounds__(256) void attn_cache_join_kernel(DsqAttnCacheArgs a, int slots)
{
    __shared__ float part[4][128], tops[4], sums[4];
    const int lane = threadIdx.x & 63, wave = wave_number();
    const int t = blockIdx.x / a.q_heads, head = blockIdx.x % a.q_heads, group = a.q_heads / a.kv_heads, most_rows = a.max_rows * group;
    int s = t;
    if (a.q_starts) {
        s = find_sequence(a.q_starts, a.rows, a.sequences, 0, t);
        if (s < 0) return;
    }
    const int t0 = a.q_starts ? clamped(a.q_starts[s], a.rows) : s, tokens = a.q_starts ? clamped(a.q_starts[s + 1], a.rows) - t0 : 1;
    if (t < t0 || t - t0 >= tokens || t - t0 >= a.max_rows) return;
    const int units = chunk_units(a, slots, lane), length = length_of(a, s), chunk = units * kUnit;
    if (length <= chunk) return;
    int of = s;
    const int slot0 = first_chunk(a, units, -1, of), chunks = (length + chunk - 1) / chunk;
    const int64_t step = (int64_t)a.kv_heads * most_rows;
    const int64_t place = slot0 * step + (int64_t)(head / group) * most_rows + (t - t0) * group + head % group;
    const float *logs = a.partial + (int64_t)(slots + a.sequences) * step * a.dim + place, *rows = a.partial + place * a.dim;

    float top = -INFINITY;
    for (int i = lane; i < chunks; i += 64) top = __builtin_elementwise_maximum(top, logs[i * step]);
    for (int off = 32; off > 0; off >>= 1) top = __builtin_elementwise_maximum(top, __shfl_xor(top, off));
    float y0 = 0.0f, y1 = 0.0f, sum = 0.0f;
    if (top != -INFINITY) {
#pragma unroll 4
        for (int i = wave; i < chunks; i += 4) {
            const float f = __builtin_amdgcn_exp2f(logs[i * step] - top);
            const float v0 = lane < a.dim ? rows[i * step * a.dim + lane] : 0.0f, v1 = lane + 64 < a.dim ? rows[i * step * a.dim + lane + 64] : 0.0f;
            sum += f;
            // (a chunk of no weight may hold NaN)
            y0 = f == 0.0f ? y0 : __builtin_fmaf(f, v0, y0);
            y1 = f == 0.0f ? y1 : __builtin_fmaf(f, v1, y1);
        }
    }
    part[wave][lane] = y0;
    part[wave][lane + 64] = y1;
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    const int d = threadIdx.x;
    if (d < a.dim) {
        const float total = sums[0] + sums[1] + sums[2] + sums[3], y = part[0][d] + part[1][d] + part[2][d] + part[3][d];
        ((E *)a.out.p)[(int64_t)t * a.out.row + head * a.out.head + d] = (E)(top == -INFINITY ? 0.0f : y / total);
    }
}

template <class E, int HD>
hipError_t launch(const DsqAttnCacheArgs &a, hipStream_t stream)
{
    const AttnCachePlan p = attn_cache_plan(a.max_rows, a.q_heads, a.kv_heads);
    const int64_t groups = (int64_t)(p.slots + a.sequences) * p.row_tiles * a.kv_heads;
    attn_cache_kernel<E, HD><<<(unsigned)groups, 256, 0, stream>>>(a, p.slots, p.row_tiles);
    if (const hipError_t e = hipGetLastError()) return e;
    attn_cache_join_kernel<E><<<(unsigned)((int64_t)a.rows * a.q_heads), 256, 0, stream>>>(a, p.slots);
    return hipGetLastError();
}

template <class E>
hipError_t of_dim(const DsqAttnCacheArgs &a, hipStream_t stream)
{
    return a.dim <= 64 ? launch<E, 64>(a, stream) : launch<E, 128>(a, stream);
}

}  // namespace

size_t dsq_attn_cache_floats(int sequences, int max_rows, int q_heads, int kv_heads, int dim)
{
    const AttnCachePlan p = attn_cache_plan(max_rows, q_heads, kv_heads);
    return (size_t)(p.slots + sequences) * max_rows * q_heads * (dim + 1);
}

hipError_t dsq_launch_attention_cache(const DsqAttnCacheArgs &a, int type, hipStream_t stream)
{
    if (type == DSQ_T_F32) return of_dim<float>(a, stream);
    if (type == DSQ_T_F16) return of_dim<_Float16>(a, stream);
    return of_dim<__bf16>(a, stream);
}
