// Attention over whole prompts, packed one behind the other, forward.
//
//   o_i = sum over visible j of p_ij v_j,  p_ij = exp(s_ij - m_i) / l_i,  s_ij = scale q_i . k_j
//
// One pass over the keys with the running maximum and sum of the softmax.  A workgroup of four waves owns 128 rows of one head, a
// wave 32 of them; tiles of keys and values go through LDS, the next tile's loads under way.  Scores are formed transposed, K Q^T,
// so that a lane holds one row's scores: maximum, sum and the factor of a raised maximum need no exchange but one between the two
// lanes of a row, and the probabilities are the second operand of V^T P^T as they lie in registers (attn_device.h).
//
// Bound by the matrix units and the vector instructions of the softmax beside them: two waves a SIMD, one's products under the other's
// exponentials.  Measured, bfloat16, 128 elements, causal: 16384 rows, 16 heads 1025 us (1073 TFLOP/s; a library product of 8192^3 reaches
// 1131; 53 % of the matrix units' cycles), 4096 rows, 32 heads 139 us (988).  float16, 64 elements, 16 sequences of up to 1000
// rows 34 us, 20 % of the matrix units' cycles: a walk over 1024 keys takes 18 by itself, and the walks do not go out by their lengths.
#include <type_traits>

#include "attn_device.h"

namespace {

// ROW_WAVES waves own 32 rows each; the others take other blocks of keys for the same rows, and their sums are joined at the end.
template <class E, int WIDTH, int ROW_WAVES>
struct Fwd {
    static constexpr int SPLIT = 4 / ROW_WAVES, ROWS = 32 * ROW_WAVES, KT = SPLIT == 1 && sizeof(E) == 2 ? 2 : 1, KEYS = 32 * KT * SPLIT;
    static constexpr int HD = kRow<WIDTH>, STEPS = WIDTH / 16, DT = WIDTH / 32, TILE = KEYS * HD;
    // binary32 keys that one wave reads alone need no LDS and no barriers: 6 % less time at 128 elements, 15 % at 96, but at 64 (where two
    // workgroups share a compute unit) 5 to 40 % more.
    static constexpr bool NEAR = sizeof(E) == 4 && ROW_WAVES == 1 && WIDTH > 64;
    // Two buffers, each a tile of keys and one of values.
    static constexpr int TILES = NEAR ? 0 : 4 * TILE * (int)sizeof(E), BYTES = most(TILES, (SPLIT - 1) * ROW_WAVES * DT * 4096);
    static constexpr bool DIRECT = sizeof(E) == 2;
    static_assert(TILES <= 131072, "tiles, and the waves' statistics beside them, fit the LDS of a compute unit");
    typedef Tile<E, HD> T;
};

// Keys of one row of a packed prompt.
template <class E>
struct PromptKeys {
    const E *k, *v;
    int64_t k_row, v_row;
    int n;
    __device__ int count() const { return n; }
    __device__ int64_t place(int j) const { return j; }
    __device__ const E *key(int64_t j) const { return k + j * k_row; }
    __device__ const E *value(int64_t j) const { return v + j * v_row; }
};

template <class E, int WIDTH, int ROW_WAVES>
__global__ __launch_bounds__(256, ROW_WAVES == 4 && (sizeof(E) == 2 || WIDTH == 64) ? 2 : 1) void attn_fwd_kernel(DsqAttnArgs a, int tiles)
{
    typedef Fwd<E, WIDTH, ROW_WAVES> F;
    typedef typename F::T T;
    typedef typename Operand<E>::type V8;
    __shared__ __align__(16) char room[F::BYTES];
    __shared__ float stat[2][F::SPLIT][F::ROWS];

    // heads that share keys meet on one of the eight dies, which take workgroups in turn
    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), r = lane & 31, h = lane >> 5, part = wave / ROW_WAVES;
    const int of = blockIdx.x / a.q_heads, turn = blockIdx.x % a.q_heads;
    const int head = a.q_heads % 8 == 0 ? turn % 8 * (a.q_heads / 8) + turn / 8 : turn;
    const int kv = head / (a.q_heads / a.kv_heads);
    const int number = attn_tile_of_turn(of, tiles, a.sequences);
    if (number < 0) return;
    const Sequence s = tile_of(a.q_starts, a.k_starts, a.q_rows, a.k_rows, a.sequences, false, F::ROWS, number);
    if (s.at < 0) return;

    const E *kp = (const E *)a.k.p + s.k0 * a.k.row + kv * a.k.head, *vp = (const E *)a.v.p + s.k0 * a.v.row + kv * a.v.head;
    const int last = s.at + F::ROWS < s.q_len ? s.at + F::ROWS - 1 : s.q_len - 1;
    const int k_end = visible(s, a.causal, last), count = (k_end + F::KEYS - 1) / F::KEYS;

    const int first_row = s.at + wave % ROW_WAVES * 32, row = first_row + r;     // this lane's row
    const bool there = row < s.q_len;
    const E *qp = (const E *)a.q.p + (int64_t)(s.q0 + row) * a.q.row + head * a.q.head;
    V8 q[F::STEPS];
#pragma unroll
    for (int i = 0; i < F::STEPS; ++i) q[i] = load_unit8(qp, 2 * i + h, a.dim, there);
    const int seen = there ? visible(s, a.causal, row) : 0;
    // keys that all of the wave's rows see, and that any does
    const int last_row = first_row + 31 < s.q_len ? first_row + 31 : s.q_len - 1;
    const int whole = first_row + 31 < s.q_len ? visible(s, a.causal, first_row) : 0;
    const int any = first_row < s.q_len ? visible(s, a.causal, last_row) : 0;

    Feed<E, F::HD, F::KEYS, F::DIRECT> km, vm;
    const auto start = [&](int t, int b) {
        E *const to = reinterpret_cast<E *>(room) + b * 2 * F::TILE;
        km.start(to, kp, a.k.row, t * F::KEYS, k_end, a.dim);
        vm.start(to + F::TILE, vp, a.v.row, t * F::KEYS, k_end, a.dim);
    };
    const float c = a.scale * kLog2e;
    float m = kNoKey, l = 0.0f;
    v16f o[F::DT];
#pragma unroll
    for (int d = 0; d < F::DT; ++d) o[d] = zeros();
    const auto hide = [&](auto &x, int at) {
        constexpr int KT = sizeof(x) / sizeof(v16f);
        if (at + 32 * KT <= whole) return;
        stay_a_branch();
        const int left = seen - at - 4 * h;
#pragma unroll
        for (int n = 0; n < KT; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[n][i] = n * 32 + 8 * (i / 4) + i % 4 < left ? x[n][i] : -INFINITY;
    };
    // one block of keys, in a buffer whose place the compiler knows
    const auto block = [&](int t, auto buffer) {
        constexpr int B = decltype(buffer)::value;
        E *const kt = reinterpret_cast<E *>(room) + B * 2 * F::TILE, *const vt = kt + F::TILE;
        km.finish(kt);
        vm.finish(vt);
        __syncthreads();
        if (t + 1 < count) start(t + 1, 1 - B);
        const int at = t * F::KEYS + part * 32 * F::KT, in = part * 32 * F::KT;      // the wave's first key, and its place in the tile
        if (at < any)
            attend<E, WIDTH, F::KT>(kt, vt, in, q, c, m, l, o, lane, [&](v16f (&x)[F::KT]) { hide(x, at); });
    };
    if constexpr (F::NEAR) {
        // each operand of the next block is sent for when this block's has been used
        RowOperands<WIDTH> ks;
        ColumnOperands<WIDTH> vs;
        if (part * 32 < any) {
            ks.fetch(kp, a.k.row, part * 32, k_end, a.dim, lane);
            vs.fetch(vp, a.v.row, part * 32, k_end, a.dim, lane);
        }
        for (int at = part * 32; at < any; at += F::KEYS) {
            const int next = at + F::KEYS < any ? at + F::KEYS : at;
            attend_to<E, WIDTH, 1>([&](int, int i) { return ks.at[i]; }, [&](int, int half, int d) { return vs.at[half][d]; }, q, c, m, l, o,
                                   [&](v16f (&x)[1]) {
                                       ks.fetch(kp, a.k.row, next, k_end, a.dim, lane);
                                       hide(x, at);
                                   });
            vs.fetch(vp, a.v.row, next, k_end, a.dim, lane);
        }
    } else {
        if (count > 0) start(0, 0);
        for (int t = 0; t < count; t += 2) {
            block(t, std::integral_constant<int, 0>());
            if (t + 1 < count) block(t + 1, std::integral_constant<int, 1>());
        }
    }

    l = both_sum(l);
    if (F::SPLIT > 1) {
        // the waves' sums to one reference, then together
        const int mine = wave % ROW_WAVES * 32 + r;
        if (h == 0) stat[0][part][mine] = m;
        __syncthreads();
        float top = m;
#pragma unroll
        for (int p = 0; p < F::SPLIT; ++p) top = __builtin_elementwise_maximum(top, stat[0][p][mine]);
        const float f = __builtin_amdgcn_exp2f(m - top);
        m = top;
        l *= f;
        if (h == 0) stat[1][part][mine] = l;
#pragma unroll
        for (int d = 0; d < F::DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] *= f;
        join<F::DT>(o, reinterpret_cast<float *>(room), wave % ROW_WAVES, ROW_WAVES, part, F::SPLIT, lane);
        if (part > 0) return;
        l = 0.0f;
#pragma unroll
        for (int p = 0; p < F::SPLIT; ++p) l += stat[1][p][mine];
    }
    const float inv = seen > 0 ? 1.0f / l : 0.0f;
    float probe = 0.0f;                      // NaN once an element is not finite
    E *op = (E *)a.out.p + (int64_t)(s.q0 + row) * a.out.row + head * a.out.head;
#pragma unroll
    for (int d = 0; d < F::DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            Side<E, 4> v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float y = seen > 0 ? o[d][4 * i + e] * inv : 0.0f;
                probe = __builtin_fmaf(y, 0.0f, probe);
                v.at[e] = (E)y;
            }
            const int at = d * 32 + 8 * i + 4 * h;
            if (there && at < a.dim) store_side(op + at, v);
        }
    if (a.lse && there && h == 0) a.lse[(int64_t)head * a.q_rows + s.q0 + row] = seen > 0 ? (m + __builtin_amdgcn_logf(l * kSumDrop<E>)) * kLn2 : -INFINITY;

    // (attn_device.h: rows that are not finite.)
    const bool asks = probe != 0.0f && there, odd = !is_finite(l);
    if (__builtin_expect(!__any(asks), 1)) return;
    const auto rows_of = [](uint64_t lanes) { return (uint32_t)(lanes | lanes >> 32); };
    const auto keys_of = [&](int i) { return PromptKeys<E>{kp, vp, a.k.row, a.v.row, visible(s, a.causal, first_row + i)}; };
    const auto query_of = [&](int i) { return (const E *)a.q.p + (int64_t)(s.q0 + first_row + i) * a.q.row + head * a.q.head; };
    const auto out_of = [&](int i) { return (E *)a.out.p + (int64_t)(s.q0 + first_row + i) * a.out.row + head * a.out.head; };
    uint32_t again = a.dim < WIDTH ? rows_of(__ballot(asks && odd)) : 0;
    if (again) {
        // Elements past a head's are its first ones again, so a key's minus infinity, a score like others, became NaN there.  A NaN in a key that all these rows
        // see explains them; a row with one in its query ends at its first keys.
        const int first = __ffs(again) - 1;
        AtOnce<E> query;
        query.load([&](int) { return query_of(first); }, a.dim);
        if (!__any(query.low[0] != query.low[0] || query.high[0] != query.high[0]) && nan_among<E>(keys_of(first), a.dim)) again = 0;
    }
    const auto put = [&](int i, const float (&y)[2]) {
        E *to = out_of(i);
        if (lane < a.dim) to[lane] = (E)y[0];
        if (lane + 64 < a.dim) to[lane + 64] = (E)y[1];
    };
    if (const uint32_t rows = rows_of(__ballot(asks && !odd))) {
        __threadfence_block();                                   // (lanes read what others of the wave have stored)
        const auto row_of = [&](int i, float (&y)[2]) {
            const E *from = out_of(i);
            y[0] = lane < a.dim ? (float)from[lane] : 0.0f, y[1] = lane + 64 < a.dim ? (float)from[lane + 64] : 0.0f;
        };
        again |= rows_to_form<E>(rows, a.dim, keys_of(__ffs(rows) - 1).n, row_of, keys_of, put);
    }
    while (again) {
        const int i = __ffs(again) - 1;
        again &= again - 1;
        float y[2];
        const float log2 = row_again<E>(query_of(i), a.dim, c, keys_of(i), y);
        put(i, y);
        if (a.lse && lane == 0) a.lse[(int64_t)head * a.q_rows + s.q0 + first_row + i] = log2 * kLn2;
    }
}

template <class E, int WIDTH, int ROW_WAVES>
hipError_t launch(const DsqAttnArgs &a, hipStream_t stream)
{
    const int rows = Fwd<E, WIDTH, ROW_WAVES>::ROWS, tiles = attn_tiles(a.q_rows, rows, a.sequences, a.q_starts);
    attn_fwd_kernel<E, WIDTH, ROW_WAVES><<<(unsigned)((int64_t)attn_turns(tiles, a.sequences) * a.q_heads), 256, 0, stream>>>(a, tiles);
    return hipGetLastError();
}

template <class E, int WIDTH>
hipError_t of_rows(const DsqAttnArgs &a, hipStream_t stream)
{
    return attn_fwd_rows(sizeof(E), WIDTH, a.q_rows, a.q_heads) == 32 ? launch<E, WIDTH, 1>(a, stream) : launch<E, WIDTH, 4>(a, stream);
}

template <class E>
hipError_t of_dim(const DsqAttnArgs &a, hipStream_t stream)
{
    switch (attn_width(a.dim)) {
    case 64: return of_rows<E, 64>(a, stream);
    case 96: return of_rows<E, 96>(a, stream);
    default: return of_rows<E, 128>(a, stream);
    }
}

}  // namespace

hipError_t dsq_launch_attention(const DsqAttnArgs &a, int type, hipStream_t stream)
{
    if (type == DSQ_T_F32) return of_dim<float>(a, stream);
    if (type == DSQ_T_F16) return of_dim<_Float16>(a, stream);
    return of_dim<__bf16>(a, stream);
}
