// Attention of single tokens, and of trees of drafted tokens, over a paged cache.
//
// The rows of a key head are the drafted tokens of a sequence times the query heads that share it.  A sequence's keys are cut into
// chunks of one length for all sequences, so that a batch of many lengths fills the card evenly, and a workgroup takes a chunk of a
// key head.  Up to 32 rows are one tile: the waves take blocks of 32 keys in turn, each with the running maximum and sum of a
// softmax, and join in LDS; a block goes through LDS of the wave's own, so a wave waits for nothing but its own loads.  Of
// more rows each of four waves takes 32, over tiles of keys that they share.  A sequence of one chunk is finished there; the others
// leave normed rows and the logarithms of their sums, which a second kernel joins.
//
// Bound by memory: every key and value is read once a key head (once for each 128 rows of it).  Measured, bfloat16, 128 elements: 32
// sequences of up to 8192 keys, 503 MB, 104 us and 6 for the join (4.8 TB/s; a large copy reaches 5.07); one of 131072 keys, 268 MB,
// 53 + 8; one of 500 keys, one launch, 9.1: a chain of dependent loads (length, page, keys, values).  float16, 8 trees of 48 drafted
// tokens, up to 4096 keys, 53 + 11: two tiles of rows read the same keys, and a chunk is a few tiles long.  binary32, one sequence of
// 131072 keys, 1.07 GB, 280 us (3.8 TB/s: one workgroup a compute unit).  256 to 16384 sequences of 256 keys 4.0 to 4.1 TB/s: every
// workgroup looks at the lengths of all sequences, which does not show.  2048 rows over 8192 keys 374 us.
#include "attn_cache_plan.h"
#include "attn_device.h"

namespace {

__device__ __forceinline__ int sum_to(int v, int lane)
{
    for (int off = 1; off < 64; off <<= 1) {
        const int u = __shfl_up(v, off);
        if (lane >= off) v += u;
    }
    return v;
}

__device__ __forceinline__ int length_of(const DsqAttnCacheArgs &a, int s) { return clamped(a.lengths[s], a.table_pages << a.page_bits); }

// The sums over the sequences that chunks are numbered by (attn_cache_plan.h).  Finds the sequence of chunk `number`, or (`number`
// negative) takes the sequence s; returns its first number, and the units of a chunk.  All 64 lanes take part; s is negative if there is none.
__device__ __forceinline__ int first_chunk(const DsqAttnCacheArgs &a, int slots, int number, int &s, int &units)
{
    const int lane = threadIdx.x & 63;
    const auto units_of = [&](int i) { return i < a.sequences ? attn_units(length_of(a, i)) : 0; };
    const int head = units_of(lane), head_sum = sum_to(head, lane);      // (the first 64 are looked at once)
    int total = __shfl(head_sum, 63);
    if (a.sequences > 64) {
        int more = 0;
        for (int i = lane + 64; i < a.sequences; i += 64) more += units_of(i);
        for (int off = 32; off > 0; off >>= 1) more += __shfl_xor(more, off);
        total += more;
    }
    units = attn_chunk_units(total, slots);
    int before = 0, found = -1, at = -1;
    for (int base = 0; base < a.sequences; base += 64) {
        const int i = base + lane, mine = base ? units_of(i) : head, sum = base ? sum_to(mine, lane) : head_sum;
        const int slot = attn_first_chunk(before + sum - mine, units, i);
        const uint64_t ok = __ballot(i < a.sequences && (number < 0 ? i <= s : slot <= number));
        if (ok == 0) break;
        const int last = 63 - __clzll((long long)ok);
        found = base + last;
        at = __shfl(slot, last);
        before += __shfl(sum, 63);
        if (last < 63) break;
    }
    s = __builtin_amdgcn_readfirstlane(found);
    units = __builtin_amdgcn_readfirstlane(units);
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
    __device__ int64_t place(int j) const { return tree.mask(first + j) & 1 ? pages.row(first + j) : -1; }
    __device__ const E *key(int64_t place) const { return k + place * dim; }
    __device__ const E *value(int64_t place) const { return v + place * dim; }
};

// What a workgroup has to do: a chunk of a sequence's keys for a key head.
struct Work {
    int s, first, end, length, tokens, mine, t0;   // keys first .. end - 1; rows: `mine` of its `tokens` from row t0 on
    bool whole;                                    // the sequence has no other chunk
    __device__ __forceinline__ void of_sequence(const DsqAttnCacheArgs &a)
    {
        length = length_of(a, s);
        t0 = a.q_starts ? clamped(a.q_starts[s], a.rows) : s;
        tokens = a.q_starts ? clamped(a.q_starts[s + 1], a.rows) - t0 : 1;
        mine = tokens < a.max_rows ? tokens : a.max_rows;
    }
    // slots: chunks that all keys are cut into; none: a workgroup takes all keys of a sequence
    __device__ __forceinline__ bool find(const DsqAttnCacheArgs &a, int slots, int number)
    {
        if (slots == 0) {
            s = number;
            of_sequence(a);
            first = 0;
            end = length;
            whole = true;
            return true;
        }
        int units;
        const int slot0 = first_chunk(a, slots, number, s, units);
        if (s < 0) return false;
        const int chunk = attn_chunk_keys(units);
        of_sequence(a);
        if ((int64_t)(number - slot0) * chunk >= length && number != slot0) return false;
        first = (number - slot0) * chunk;
        end = length - first < chunk ? length : first + chunk;
        whole = length <= chunk;
        return true;
    }
};

// Where the logarithms of a row's chunks lie side by side, behind all rows: [kv heads][rows][chunks].
__device__ __forceinline__ float *logs_of(const DsqAttnCacheArgs &a, int slots, int kv, int of)
{
    const int64_t most_rows = (int64_t)a.max_rows * (a.q_heads / a.kv_heads), chunks = slots + a.sequences;
    return a.partial + chunks * a.kv_heads * most_rows * a.dim + (kv * most_rows + of) * chunks;
}

// A finished row (its logarithm to base 2, normed elements lane and lane + 64 of a wave): to the output, or to where chunks are joined.
template <class E>
__device__ __forceinline__ void leave_row(const DsqAttnCacheArgs &a, const Work &w, int slots, int number, int kv, int of, int token, bool seen, float log2, const float y[2])
{
    const int lane = threadIdx.x & 63, group = a.q_heads / a.kv_heads, most_rows = a.max_rows * group;
    if (w.whole) {
        E *to = (E *)a.out.p + (int64_t)(w.t0 + token) * a.out.row + (kv * group + of - token * group) * a.out.head;
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (lane + 64 * e < a.dim) to[lane + 64 * e] = (E)y[e];
        return;
    }
    // (a row whose scores are all -inf is NaN by the formula, but only where no other chunk has more)
    if (!(log2 > kNoKey) && log2 == log2) log2 = kNoKey;
    const int64_t place = ((int64_t)number * a.kv_heads + kv) * most_rows + of;
#pragma unroll
    for (int e = 0; e < 2; ++e)
        if (lane + 64 * e < a.dim) a.partial[place * a.dim + lane + 64 * e] = y[e];
    if (lane == 0) logs_of(a, slots, kv, of)[number] = seen ? log2 : -INFINITY;
}

// The keys of a chunk that a token sees.
template <class E>
__device__ __forceinline__ CacheKeys<E> keys_of(const DsqAttnCacheArgs &a, const Work &w, const Pages &pages, int token)
{
    const Tree its = {a.tree ? a.tree + (int64_t)(w.t0 + token) * a.tree_words : nullptr, a.tree_words, token, w.length - w.tokens};
    return {(const E *)a.k_cache, (const E *)a.v_cache, pages, its, w.first, w.end - w.first, a.dim};
}

template <class E>
__device__ __forceinline__ float again(const DsqAttnCacheArgs &a, const Work &w, const CacheKeys<E> &keys, int kv, int of, int token, float c, float y[2])
{
    const int head = kv * (a.q_heads / a.kv_heads) + of - token * (a.q_heads / a.kv_heads);
    return row_again<E>((const E *)a.q.p + (int64_t)(w.t0 + token) * a.q.row + head * a.q.head, a.dim, c, keys, y);
}

// Puts -inf in the place of the scores of 32 keys whose bit is not set.
__device__ __forceinline__ void hide_keys(v16f &x, uint32_t mask, int h)
{
    if (!__any(mask != 0xffffffffu)) return;
    stay_a_branch();
    mask >>= 4 * h;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = mask >> (8 * (i / 4) + i % 4) & 1 ? x[i] : -INFINITY;
}

// ---- up to 32 rows: WAVES waves take blocks of 32 keys in turn ------------------------------------------

template <class E, int WIDTH, int WAVES>
__global__ __launch_bounds__(64 * WAVES, sizeof(E) == 2 ? 2 : 1) void attn_cache_kernel(DsqAttnCacheArgs a, int slots)
{
    constexpr int HD = kRow<WIDTH>, STEPS = WIDTH / 16, DT = WIDTH / 32;
    typedef Tile<E, HD> T;
    typedef typename Operand<E>::type V8;
    constexpr int PIECES = 32 * T::UNITS / 64, STRIDE = 32 * WAVES, WAVE_BYTES = most(32 * HD * 4, 64 * HD * (int)sizeof(E));
    __shared__ __align__(16) char room[WAVES * WAVE_BYTES];
    __shared__ float stat[WAVES][2][32];
    __shared__ uint32_t seen_by[WAVES][32];

    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), r = lane & 31, h = lane >> 5;
    const int number = blockIdx.x / a.kv_heads, kv = blockIdx.x % a.kv_heads, group = a.q_heads / a.kv_heads;
    Work w;
    if (!w.find(a, slots, number)) return;
    const Pages pages = {a.table + w.s * a.table_row, a.pages, a.table_pages, a.page_bits, kv, a.kv_heads, w.length};
    const E *kp = (const E *)a.k_cache, *vp = (const E *)a.v_cache;
    int j = w.first + wave * 32;
    int64_t next = j < w.end ? pages.row(j + r) : -1;
    if (w.mine <= 0) return;

    const int token = r / group, head = kv * group + r % group;
    const bool there = token < w.mine;
    const Tree tree = {a.tree && there ? a.tree + (int64_t)(w.t0 + token) * a.tree_words : nullptr, a.tree_words, token, w.length - w.tokens};

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
    if (j < w.end) fetch(next);
    next = j + STRIDE < w.end ? pages.row(j + STRIDE + r) : -1;
    V8 q[STEPS];
    const E *qp = (const E *)a.q.p + (int64_t)(w.t0 + token) * a.q.row + head * a.q.head;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) q[i] = load_unit8(qp, 2 * i + h, a.dim, there);

    const float c = a.scale * kLog2e;
    float m = kNoKey, l = 0.0f;
    uint32_t any = 0;
    v16f o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = zeros();
    for (; j < w.end; j += STRIDE) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int piece = lane + 64 * i, at = T::place(piece / T::UNITS, piece % T::UNITS);
            *reinterpret_cast<v4u *>(ks + at) = kr[i];
            *reinterpret_cast<v4u *>(vs + at) = vr[i];
        }
        wave_order();
        const uint32_t mask = valid & (there ? tree.mask(j) : 0);
        if (j + STRIDE < w.end) {
            fetch(next);
            next = j + 2 * STRIDE < w.end ? pages.row(j + 2 * STRIDE + r) : -1;
        }
        any |= mask;
        attend<E, WIDTH, 1>(ks, vs, 0, q, c, m, l, o, lane, [&](v16f (&x)[1]) { hide_keys(x[0], mask, h); });
        wave_order();
    }

    // ---- the waves' rows, in the room of their tiles: 16-byte units exchanged within a row by its number
    const int rows = w.mine * group < 32 ? w.mine * group : 32;
    float *mine_o = reinterpret_cast<float *>(room + wave * WAVE_BYTES);
    if (r < rows) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<v4f *>(mine_o + r * HD + ((d * 8 + 2 * i + h) ^ (r % (HD / 4))) * 4) =
                    v4f{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
    }
    l = both_sum(l);
    if (h == 0) {
        stat[wave][0][r] = m;
        stat[wave][1][r] = l;
        seen_by[wave][r] = any;
    }
    __syncthreads();
    for (int i = wave; i < rows; i += WAVES) {
        float top = kNoKey;
        uint32_t seen = 0;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) top = __builtin_elementwise_maximum(top, stat[v][0][i]), seen |= seen_by[v][i];
        float f[WAVES], sum = 0.0f;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) {
            f[v] = __builtin_amdgcn_exp2f(stat[v][0][i] - top);
            sum = __builtin_fmaf(stat[v][1][i], f[v], sum);
        }
        float y[2];
        bool bad = false;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int d = lane + 64 * e;
            y[e] = 0.0f;
            if (d < WIDTH) {
#pragma unroll
                for (int v = 0; v < WAVES; ++v)
                    y[e] = __builtin_fmaf(reinterpret_cast<const float *>(room + v * WAVE_BYTES)[i * HD + ((d / 4) ^ (i % (HD / 4))) * 4 + d % 4], f[v], y[e]);
                y[e] = seen ? y[e] / sum : 0.0f;
            }
            bad |= !is_finite(y[e]);
        }
        float log2 = top + __builtin_amdgcn_logf(sum * kSumDrop<E>);
        if (__builtin_expect(__any(bad) && is_finite(sum), 0)) {
            const CacheKeys<E> keys = keys_of<E>(a, w, pages, i / group);
            const Spoilt its = spoilt_of(y[0], y[1]);
            float z[2] = {0.0f, 0.0f};
            if (!its.explained_by(add_spoilt<E>(keys, 0, a.dim, its, z))) {
                if (stands_for(z, its)) y[0] = is_finite(z[0]) ? y[0] : z[0], y[1] = is_finite(z[1]) ? y[1] : z[1];
                else log2 = again<E>(a, w, keys, kv, i, i / group, c, y);
            }
        }
        leave_row<E>(a, w, slots, number, kv, i, i / group, seen != 0, log2, y);
    }
}

// ---- more rows: four waves take 32 each, over tiles of keys that they share ------------------------------------

template <class E, int WIDTH>
__global__ __launch_bounds__(256, sizeof(E) == 2 ? 2 : 1) void attn_cache_tiles_kernel(DsqAttnCacheArgs a, int slots, int row_tiles)
{
    constexpr int HD = kRow<WIDTH>, STEPS = WIDTH / 16, DT = WIDTH / 32;
    typedef Tile<E, HD> T;
    typedef typename Operand<E>::type V8;
    constexpr int KT = sizeof(E) == 2 ? 2 : 1, KEYS = 32 * KT, TILE = KEYS * HD;
    constexpr int PIECES = KEYS * T::UNITS / 256, STEP = 256 / T::UNITS;
    __shared__ __align__(16) E tiles_at[2][2][TILE];
    __shared__ uint32_t there_at[2][KT];
    static_assert(32 * HD * 4 <= (int)sizeof(E) * TILE, "a wave's rows fit a tile");

    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), r = lane & 31, h = lane >> 5;
    const int kv = blockIdx.x % a.kv_heads, number = blockIdx.x / a.kv_heads / row_tiles, rt = blockIdx.x / a.kv_heads % row_tiles;
    const int group = a.q_heads / a.kv_heads;
    Work w;
    if (!w.find(a, slots, number) || rt * 128 >= w.mine * group) return;
    const Pages pages = {a.table + w.s * a.table_row, a.pages, a.table_pages, a.page_bits, kv, a.kv_heads, w.length};
    const E *kp = (const E *)a.k_cache, *vp = (const E *)a.v_cache;

    const int row0 = rt * 128 + wave * 32, row = row0 + r, token = row / group, head = kv * group + row % group;
    const bool there = token < w.mine, busy = row0 < w.mine * group;
    const Tree tree = {a.tree && there ? a.tree + (int64_t)(w.t0 + token) * a.tree_words : nullptr, a.tree_words, token, w.length - w.tokens};
    V8 q[STEPS];
    const E *qp = (const E *)a.q.p + (int64_t)(w.t0 + token) * a.q.row + head * a.q.head;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) q[i] = load_unit8(qp, 2 * i + h, a.dim, there);

    // A thread moves 16 bytes of the rows tid / UNITS + STEP i of a tile; a place is looked up one tile before its load.  Where pages
    // hold whole tiles, there is one place for all.
    const int u = tid % T::UNITS, from = tid / T::UNITS;
    const bool one = (1 << a.page_bits) >= KEYS;
    v4u kr[PIECES], vr[PIECES];
    int64_t place[PIECES];
    auto look = [&](int j) {
        if (one) {
            place[0] = j < w.end ? pages.row(j) : -1;
            return;
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) place[i] = j + from + STEP * i < w.end ? pages.row(j + from + STEP * i) : -1;
    };
    uint32_t valid = 0;                      // bit i: of piece i
    const auto load = [&](const E *p, int64_t at, bool ok) {
        return ok && u * T::PER < a.dim ? *reinterpret_cast<const v4u *>(p + at * a.dim + u * T::PER) : v4u{0, 0, 0, 0};
    };
    auto fetch = [&](int j) {
        valid = 0;
        if (one) {
            const int64_t first = (int64_t)__builtin_amdgcn_readfirstlane((int)(place[0] >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)place[0]);
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int row = from + STEP * i;
                const bool ok = first >= 0 && j + row < w.end;
                valid |= (ok ? 1u : 0u) << i;
                kr[i] = load(kp + first * a.dim, row, ok);
                vr[i] = load(vp + first * a.dim, row, ok);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            valid |= (place[i] >= 0 ? 1u : 0u) << i;
            kr[i] = load(kp, place[i], place[i] >= 0);
            vr[i] = load(vp, place[i], place[i] >= 0);
        }
    };

    const float c = a.scale * kLog2e;
    float m = kNoKey, l = 0.0f;
    uint32_t any = 0;
    v16f o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = zeros();
    look(w.first);
    fetch(w.first);
    look(w.first + KEYS);
    if (tid < 2 * KT) there_at[tid / KT][tid % KT] = 0;
    __syncthreads();
    int b = 0;
    for (int j = w.first; j < w.end; j += KEYS, b ^= 1) {
        E *const kt = tiles_at[b][0], *const vt = tiles_at[b][1];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int at = T::place(from + STEP * i, u), key = from + STEP * i;
            *reinterpret_cast<v4u *>(kt + at) = kr[i];
            *reinterpret_cast<v4u *>(vt + at) = vr[i];
            if (u == 0 && (valid >> i & 1)) atomicOr(&there_at[b][key / 32], 1u << key % 32);
        }
        __syncthreads();
        uint32_t mask[KT];
#pragma unroll
        for (int n = 0; n < KT; ++n) mask[n] = there_at[b][n] & (there ? tree.mask(j + n * 32) : 0);
        if (j + KEYS < w.end) {
            fetch(j + KEYS);
            look(j + 2 * KEYS);
        }
#pragma unroll
        for (int n = 0; n < KT; ++n) any |= mask[n];
        if (busy)
            attend<E, WIDTH, KT>(kt, vt, 0, q, c, m, l, o, lane, [&](v16f (&x)[KT]) {
#pragma unroll
                for (int n = 0; n < KT; ++n) hide_keys(x[n], mask[n], h);
            });
        // (the other buffer's bits are read before the barrier that comes, and set after it)
        if (tid < KT) there_at[b ^ 1][tid] = 0;
        __syncthreads();
    }
    if (!busy) return;

    // The rows lie transposed in registers: through LDS, a wave's in the room of its tile (units exchanged as in a tile).
    float *mine_o = reinterpret_cast<float *>(&tiles_at[0][0][0]) + wave * TILE * (int)sizeof(E) / 4;
    l = both_sum(l);
    const float inv = any ? 1.0f / l : 0.0f, log2 = m + __builtin_amdgcn_logf(l * kSumDrop<E>);
    float probe = 0.0f;                      // NaN once an element is not finite
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v4f y = {0.0f, 0.0f, 0.0f, 0.0f};
            if (any) y = v4f{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]} * inv;
#pragma unroll
            for (int e = 0; e < 4; ++e) probe = __builtin_fmaf(y[e], 0.0f, probe);
            *reinterpret_cast<v4f *>(mine_o + r * HD + ((d * 8 + 2 * i + h) ^ (r % (HD / 4))) * 4) = y;
        }
    wave_order();
    const int most_rows = a.max_rows * group;
    const int64_t rows_at = ((int64_t)number * a.kv_heads + kv) * most_rows + row0;
    constexpr int ACROSS = HD / 4, DOWN = 64 / ACROSS;          // lanes of a row, rows of a step
    int of_lane = lane;
    asm volatile("" : "+v"(of_lane));        // (its rows' numbers are not kept from before the loop, whose registers are full)
#pragma unroll
    for (int i = 0; i < 32; i += DOWN) {
        const int its = i + of_lane / ACROSS, at = of_lane % ACROSS;
        const v4f y = *reinterpret_cast<const v4f *>(mine_o + its * HD + (at ^ (its % (HD / 4))) * 4);
        const int of = row0 + its;
        if (of >= w.mine * group || at * 4 >= a.dim) continue;
        if (w.whole) {
            Side<E, 4> v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v.at[e] = (E)y[e];
            store_side((E *)a.out.p + (int64_t)(w.t0 + of / group) * a.out.row + (kv * group + of % group) * a.out.head + at * 4, v);
        } else {
            *reinterpret_cast<v4f *>(a.partial + (rows_at + its) * a.dim + at * 4) = y;
        }
    }
    if (!w.whole && there && h == 0) logs_of(a, slots, kv, row)[number] = any ? log2 > kNoKey || log2 != log2 ? log2 : kNoKey : -INFINITY;
    // (rows whose sum is not finite see a score that is none; the keys before the drafted ones are seen by all)
    const uint64_t asks = __ballot(probe != 0.0f && there && is_finite(l));
    if (__builtin_expect(asks == 0, 1)) return;
    const int before = w.length - w.tokens - w.first, keys = w.end - w.first;
    const auto token_of = [&](int i) { return __builtin_amdgcn_readlane(token, i); };
    const auto keys_of_row = [&](int i) { return keys_of<E>(a, w, pages, token_of(i)); };
    const auto row_of = [&](int i, float (&y)[2]) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int d = of_lane + 64 * e;
            y[e] = d < a.dim ? mine_o[i * HD + ((d / 4) ^ (i % (HD / 4))) * 4 + d % 4] : 0.0f;
        }
    };
    uint32_t rows = rows_to_form<E>((uint32_t)(asks | asks >> 32), a.dim, before < 0 ? 0 : before < keys ? before : keys, row_of, keys_of_row,
                                    [&](int i, const float (&y)[2]) { leave_row<E>(a, w, slots, number, kv, row0 + i, token_of(i), true, lanes_number(log2, i), y); });
    while (rows) {
        const int i = __ffs(rows) - 1;
        rows &= rows - 1;
        float y[2];
        const float its = again<E>(a, w, keys_of_row(i), kv, row0 + i, token_of(i), c, y);
        leave_row<E>(a, w, slots, number, kv, row0 + i, token_of(i), true, its, y);
    }
}

// The chunks of a row, weighted by their shares of its sum (before they are added: values near the end of binary32 stay inside it).  WAVES
// waves take the chunks of a row in turn, or (WAVES = 1) a wave takes HEADS heads at once.
template <class E, int WAVES, int HEADS>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void attn_cache_join_kernel(DsqAttnCacheArgs a, int slots)
{
    static_assert(WAVES == 1 || HEADS == 1, "");
    constexpr int AT_ONCE = HEADS == 1 ? 8 : 4;
    __shared__ float part[WAVES == 1 ? 1 : WAVES][128];
    const int lane = threadIdx.x & 63, wave = wave_number(), group = a.q_heads / a.kv_heads, most_rows = a.max_rows * group;
    const int turns = (a.q_heads + HEADS - 1) / HEADS;
    const int64_t unit = WAVES == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
    const int t = (int)(unit / turns), head0 = (int)(unit % turns) * HEADS, turn = WAVES == 1 ? 0 : wave;
    if (t >= a.rows) return;
    int s = t, units;
    if (a.q_starts) s = find_sequence(a.q_starts, a.rows, a.sequences, 0, t);
    if (s < 0) return;
    int of = s;
    const int slot0 = first_chunk(a, slots, -1, of, units);
    const int t0 = a.q_starts ? clamped(a.q_starts[s], a.rows) : s, tokens = a.q_starts ? clamped(a.q_starts[s + 1], a.rows) - t0 : 1;
    const int length = length_of(a, s), chunk = attn_chunk_keys(units), chunks = (int)(((int64_t)length + chunk - 1) / chunk);
    if (t < t0 || t - t0 >= tokens || t - t0 >= a.max_rows || chunks <= 1) return;
    const int64_t step = (int64_t)a.kv_heads * most_rows * a.dim;
    const int d0 = lane < a.dim ? lane : 0, d1 = lane + 64 < a.dim ? lane + 64 : 0;
    const float *logs[HEADS], *rows[HEADS];
    float top[HEADS], y0[HEADS], y1[HEADS], by[HEADS];
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        const int head = head0 + i < a.q_heads ? head0 + i : a.q_heads - 1, row = (t - t0) * group + head % group;
        logs[i] = logs_of(a, slots, head / group, row) + slot0;
        rows[i] = a.partial + slot0 * step + ((int64_t)(head / group) * most_rows + row) * a.dim;
        top[i] = -INFINITY;
        y0[i] = y1[i] = by[i] = 0.0f;
    }
    for (int c = 0; c < chunks; c += 64)
#pragma unroll
        for (int i = 0; i < HEADS; ++i) top[i] = __builtin_elementwise_maximum(top[i], c + lane < chunks ? logs[i][c + lane] : -INFINITY);
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        for (int off = 32; off > 0; off >>= 1) top[i] = __builtin_elementwise_maximum(top[i], __shfl_xor(top[i], off));
        top[i] = top[i] == -INFINITY ? 0.0f : top[i];            // (no chunk has a key that the row sees: all weights are zero)
    }
    for (int c = 0; c < chunks; c += 64)
#pragma unroll
        for (int i = 0; i < HEADS; ++i) by[i] += c + lane < chunks ? __builtin_amdgcn_exp2f(logs[i][c + lane] - top[i]) : 0.0f;
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        for (int off = 32; off > 0; off >>= 1) by[i] += __shfl_xor(by[i], off);
        by[i] = by[i] == 0.0f ? 0.0f : 1.0f / by[i];
    }
    for (int base = 0; base < chunks; base += 64) {
        float f[HEADS];
        const int n = chunks - base < 64 ? chunks - base : 64;
#pragma unroll
        for (int i = 0; i < HEADS; ++i) f[i] = lane < n ? __builtin_amdgcn_exp2f(logs[i][base + lane] - top[i]) * by[i] : 0.0f;
        for (int c0 = turn; c0 < n; c0 += AT_ONCE * WAVES) {
            // (loads of several chunks under way; those past the last have no weight)
            float v0[AT_ONCE][HEADS], v1[AT_ONCE][HEADS];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int c = c0 + k * WAVES < n ? c0 + k * WAVES : c0;
#pragma unroll
                for (int i = 0; i < HEADS; ++i) v0[k][i] = rows[i][(base + c) * step + d0], v1[k][i] = rows[i][(base + c) * step + d1];
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k)
#pragma unroll
                for (int i = 0; i < HEADS; ++i) {
                    const float p = c0 + k * WAVES < n ? __shfl(f[i], (c0 + k * WAVES) & 63) : 0.0f;
                    // (a chunk of no weight may hold NaN)
                    y0[i] = p == 0.0f ? y0[i] : __builtin_fmaf(p, v0[k][i], y0[i]);
                    y1[i] = p == 0.0f ? y1[i] : __builtin_fmaf(p, v1[k][i], y1[i]);
                }
        }
    }
    if (WAVES > 1) {
        part[wave][lane] = y0[0];
        part[wave][lane + 64] = y1[0];
        __syncthreads();
        if (turn > 0) return;
        y0[0] = y1[0] = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) y0[0] += part[w][lane], y1[0] += part[w][lane + 64];
    }
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        if (head0 + i >= a.q_heads) return;
        E *to = (E *)a.out.p + (int64_t)t * a.out.row + (head0 + i) * a.out.head;
        if (lane < a.dim) to[lane] = (E)y0[i];
        if (lane + 64 < a.dim) to[lane + 64] = (E)y1[i];
    }
}

template <class E, int WIDTH>
hipError_t launch(const DsqAttnCacheArgs &a, hipStream_t stream)
{
    const AttnCachePlan p = attn_cache_plan(a.max_rows, a.q_heads, a.kv_heads, a.sequences, (int64_t)a.table_pages << a.page_bits);
    const unsigned groups = (unsigned)((int64_t)(p.slots + a.sequences) * p.row_tiles * a.kv_heads);
    if (p.tiles) attn_cache_tiles_kernel<E, WIDTH><<<groups, 256, 0, stream>>>(a, p.slots, p.row_tiles);
    else if (p.single) attn_cache_kernel<E, WIDTH, sizeof(E) == 2 ? 8 : 4><<<groups, sizeof(E) == 2 ? 512 : 256, 0, stream>>>(a, p.slots);
    else attn_cache_kernel<E, WIDTH, 4><<<groups, 256, 0, stream>>>(a, p.slots);
    if (const hipError_t e = hipGetLastError()) return e;
    const int64_t rows = (int64_t)a.rows * a.q_heads, fours = (int64_t)a.rows * ((a.q_heads + 3) / 4);
    switch (attn_cache_join(p, a.rows, a.q_heads, a.sequences)) {
    case kJoinNone: break;
    case kJoinSixteen: attn_cache_join_kernel<E, 16, 1><<<(unsigned)rows, 1024, 0, stream>>>(a, p.slots); break;
    case kJoinOne: attn_cache_join_kernel<E, 1, 1><<<(unsigned)((rows + 3) / 4), 256, 0, stream>>>(a, p.slots); break;
    case kJoinFour: attn_cache_join_kernel<E, 1, 4><<<(unsigned)((fours + 3) / 4), 256, 0, stream>>>(a, p.slots); break;
    }
    return hipGetLastError();
}

template <class E>
hipError_t of_dim(const DsqAttnCacheArgs &a, hipStream_t stream)
{
    switch (attn_width(a.dim)) {
    case 64: return launch<E, 64>(a, stream);
    case 96: return launch<E, 96>(a, stream);
    default: return launch<E, 128>(a, stream);
    }
}

}  // namespace

size_t dsq_attn_cache_floats(int sequences, int max_rows, int q_heads, int kv_heads, int dim)
{
    // (the room does not go by the table's size: as many chunks as any call has)
    const AttnCachePlan p = attn_cache_plan(max_rows, q_heads, kv_heads, sequences, INT64_MAX);
    return (size_t)(p.slots + sequences) * max_rows * q_heads * (dim + 1);
}

hipError_t dsq_launch_attention_cache(const DsqAttnCacheArgs &a, int type, hipStream_t stream)
{
    if (type == DSQ_T_F32) return of_dim<float>(a, stream);
    if (type == DSQ_T_F16) return of_dim<_Float16>(a, stream);
    return of_dim<__bf16>(a, stream);
}
