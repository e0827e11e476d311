// Attention over whole prompts, backward.
//
//   p_ij = exp(s_ij - lse_i),  D_i = do_i . o_i,  ds_ij = p_ij (do_i . v_j - D_i)
//   dv_j = sum_i p_ij do_i,  dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i
//
// Two kernels, each of which forms the scores again, so that every sum has one owner and no atomics are needed: the same bits every
// time.  One owns rows of queries (D and dq), the other keys, over all heads that share them (dk and dv).  In both a
// lane holds a column of the 32x32 results, so probabilities and ds are the second operand of the next product as they lie
// in registers (attn_device.h).
//
// Seven products of the scores' size, where one kernel with atomics would have five.  Measured, bfloat16, 4 x 2048 rows, causal, 16 heads
// of 128 in four groups: queries 118 us (44 % of the matrix units' cycles), keys 195 us (34 %; LDS 35 %: one workgroup of eight waves a
// compute unit goes through its phases in step).  binary32, 80 elements, 3 sequences of up to 701 rows: 48 and 56 us, few workgroups of one wave a SIMD.
#include <type_traits>

#include "attn_device.h"

namespace {

// ds and p enter the matrix instruction in the inputs' type.  In float16 a probability below 2^-14 would lose digits: there p is taken
// times 2^10, and the sums divided by it.
template <class E>
constexpr float kLift = 0.0f;
template <>
constexpr float kLift<_Float16> = 10.0f;
template <class E>
constexpr float kDrop = 1.0f;
template <>
constexpr float kDrop<_Float16> = 0x1p-10f;

// Four consecutive elements a store: a lane's column of transposed 32x32 results as a row of the output.
template <class E, int DT>
__device__ __forceinline__ void store_row(E *to, const v16f (&o)[DT], float by, int h, int dim)
{
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            Side<E, 4> v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v.at[e] = (E)(o[d][4 * i + e] * by);
            const int at = d * 32 + 8 * i + 4 * h;
            if (at < dim) store_side(to + at, v);
        }
}

// ---- queries ------------------------------------------------------------------------------------
//
// ROW_WAVES waves own 32 rows each; the others take other blocks of 32 keys for the same rows, and their sums are joined.

template <class E, int WIDTH, int ROW_WAVES>
__global__ __launch_bounds__(256, sizeof(E) == 2 && ROW_WAVES == 4 ? 2 : 1) void attn_bwd_q_kernel(DsqAttnBwdArgs a, int tiles)
{
    constexpr int HD = kRow<WIDTH>, STEPS = WIDTH / 16, DT = WIDTH / 32;
    typedef Tile<E, HD> T;
    typedef typename Operand<E>::type V8;
    constexpr int SPLIT = 4 / ROW_WAVES, ROWS = 32 * ROW_WAVES, KT = SPLIT == 1 ? 2 : 1, KEYS = 32 * KT * SPLIT;
    constexpr int BUFFERS = SPLIT == 1 ? 2 : 1;
    constexpr int TILE = KEYS * HD, JOIN = (SPLIT - 1) * ROW_WAVES * DT * 4096;
    __shared__ __align__(16) char room[most(BUFFERS * 2 * TILE * (int)sizeof(E), JOIN)];
    __shared__ float parts[SPLIT][ROWS];
    E *const tiles_at = reinterpret_cast<E *>(room);

    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), r = lane & 31, h = lane >> 5, part = wave / ROW_WAVES;
    const int of = blockIdx.x / a.q_heads, turn = blockIdx.x % a.q_heads;
    const int head = a.q_heads % 8 == 0 ? turn % 8 * (a.q_heads / 8) + turn / 8 : turn;
    const int kv = head / (a.q_heads / a.kv_heads);
    const int number = attn_tile_of_turn(of, tiles, a.sequences);
    if (number < 0) return;
    const Sequence s = tile_of(a.q_starts, a.k_starts, a.q_rows, a.k_rows, a.sequences, false, ROWS, number);
    if (s.at < 0) return;

    const E *kp = (const E *)a.k.p + s.k0 * a.k.row + kv * a.k.head, *vp = (const E *)a.v.p + s.k0 * a.v.row + kv * a.v.head;
    const int last = s.at + ROWS < s.q_len ? s.at + ROWS - 1 : s.q_len - 1;
    const int k_end = visible(s, a.causal, last), count = (k_end + KEYS - 1) / KEYS;

    const int first_row = s.at + wave % ROW_WAVES * 32, row = first_row + r;
    const bool there = row < s.q_len;
    const int64_t token = s.q0 + row;
    const E *qp = (const E *)a.q.p + token * a.q.row + head * a.q.head, *gp = (const E *)a.grad_out.p + token * a.grad_out.row + head * a.grad_out.head;
    const E *yp = (const E *)a.out.p + token * a.out.row + head * a.out.head;
    V8 q[STEPS], g[STEPS];
    float delta = 0.0f;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        q[i] = load_unit8(qp, 2 * i + h, a.dim, there);
        g[i] = load_unit8(gp, 2 * i + h, a.dim, there);
        const V8 y = load_unit8(yp, 2 * i + h, a.dim, there);
#pragma unroll
        for (int e = 0; e < 8; ++e) delta = __builtin_fmaf((float)g[i][e], (float)y[e], delta);
    }
    delta = both_sum(delta);
    const int64_t stat = (int64_t)head * a.q_rows + token;
    const int seen = there ? visible(s, a.causal, row) : 0;
    const float lse = seen > 0 ? a.lse[stat] * kLog2e - kLift<E> : 0.0f;
    const int last_row = first_row + 31 < s.q_len ? first_row + 31 : s.q_len - 1;
    const int whole = first_row + 31 < s.q_len ? visible(s, a.causal, first_row) : 0;
    const int any = first_row < s.q_len ? visible(s, a.causal, last_row) : 0;
    const float c = a.scale * kLog2e;

    Feed<E, HD, KEYS, sizeof(E) == 2 && BUFFERS == 2> km, vm;
    const auto start = [&](int t, int b) {
        E *const to = tiles_at + b * 2 * TILE;
        km.start(to, kp, a.k.row, t * KEYS, k_end, a.dim);
        vm.start(to + TILE, vp, a.v.row, t * KEYS, k_end, a.dim);
    };
    v16f dq[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) dq[d] = zeros();
    if (count > 0) start(0, 0);
    // One block of keys, in a buffer whose place the compiler knows: p in x, grad_out . v in y, zeros for what is not seen.
    const auto scores = [&](const E *kt, const E *vt, int in, int at, v16f &x, v16f &y) {
        x = y = zeros();
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            x = multiply(T::row_operand(kt, in + r, i, h), q[i], x);
            y = multiply(T::row_operand(vt, in + r, i, h), g[i], y);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], c, -lse));
        if (at + 32 > whole) {
            stay_a_branch();
            const int left = seen - at - 4 * h;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[i] = 8 * (i / 4) + i % 4 < left ? x[i] : 0.0f;
                y[i] = 8 * (i / 4) + i % 4 < left ? y[i] : 0.0f;
            }
        }
    };
    // D is formed from the result as it was stored.  Rows of few keys have large results, whose rounding is a third of the error of all gradients
    // together: they form it again from p.
    if (sizeof(E) == 2 && k_end <= 128) {
        float sum = 0.0f;
        for (int t = 0; t < count; ++t) {
            E *const kt = tiles_at + (BUFFERS == 2 ? t & 1 : 0) * 2 * TILE, *const vt = kt + TILE;
            if (BUFFERS == 1) __syncthreads();
            km.finish(kt);
            vm.finish(vt);
            __syncthreads();
            if (t + 1 < count) start(t + 1, BUFFERS == 2 ? (t + 1) & 1 : 0);
            for (int n = 0; n < KT; ++n) {
                const int in = (part * KT + n) * 32, at = t * KEYS + in;
                if (at >= any) break;
                v16f x, y;
                scores(kt, vt, in, at, x, y);
#pragma unroll
                for (int i = 0; i < 16; ++i) sum = __builtin_fmaf(x[i], y[i], sum);
            }
        }
        sum = both_sum(sum) * kDrop<E>;
        if (SPLIT > 1) {
            if (h == 0) parts[part][wave % ROW_WAVES * 32 + r] = sum;
            __syncthreads();
            sum = 0.0f;
#pragma unroll
            for (int p = 0; p < SPLIT; ++p) sum += parts[p][wave % ROW_WAVES * 32 + r];
        }
        __syncthreads();
        delta = sum;
        if (count > 0) start(0, 0);
    }
    if (there && h == 0 && part == 0) a.delta[stat] = delta;
    delta *= kDrop<E>;
    const auto block = [&](int t, auto buffer) {
        constexpr int B = decltype(buffer)::value;
        E *const kt = tiles_at + B * 2 * TILE, *const vt = kt + TILE;
        if (BUFFERS == 1) __syncthreads();
        km.finish(kt);
        vm.finish(vt);
        __syncthreads();
        if (t + 1 < count) start(t + 1, BUFFERS - 1 - B);
#pragma unroll
        for (int n = 0; n < KT; ++n) {
            const int in = (part * KT + n) * 32, at = t * KEYS + in;     // the wave's first key, and its place in the tile
            if (at >= any) break;
            v16f x, y;
            scores(kt, vt, in, at, x, y);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] *= __builtin_fmaf(y[i], kDrop<E>, -delta);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const V8 ds = operand_of<E>(x, half);
#pragma unroll
                for (int d = 0; d < DT; ++d) dq[d] = multiply(T::column_operand(kt, in + half * 16, d * 32, lane), ds, dq[d]);
            }
        }
    };
    for (int t = 0; t < count; t += 2) {
        block(t, std::integral_constant<int, 0>());
        if (t + 1 < count) block(t + 1, std::integral_constant<int, BUFFERS - 1>());
    }
    join<DT>(dq, reinterpret_cast<float *>(room), wave % ROW_WAVES, ROW_WAVES, part, SPLIT, lane);
    if (there && part == 0) store_row<E, DT>((E *)a.grad_q.p + token * a.grad_q.row + head * a.grad_q.head, dq, a.scale, h, a.dim);
}

// ---- keys and values ------------------------------------------------------------------------------
//
// Two waves share 32 keys and blocks of 32 rows: one forms the scores and p and sums dv, the other forms grad_out . v and ds and sums dk,
// with p handed over in LDS.  Each so holds one operand and one sum in registers, has SUB blocks of rows under way at once, and another
// wave on its SIMD whose products run under its exponentials.  A workgroup has KEY_PAIRS such pairs side by side along the keys and
// ROW_PAIRS along the rows, whose sums are joined at the end.  Where there are few keys the rows are split over workgroups too, which
// leave their sums in the workspace for a kernel that adds them in order.
//
// (Measured beside it at 4 x 2048 rows, 16 heads of 128 in four groups: both waves form the scores and nothing is handed over 268 us for 224;
// one wave holds both sums and operands, one wave a SIMD, 422; one block of rows at a time 234; pairs 2 x 1 or 1 x 2, two workgroups
// a compute unit, 350 and 284.)

template <class E, int WIDTH, int KEY_PAIRS, int ROW_PAIRS, int SUB>
__global__ __launch_bounds__(128 * KEY_PAIRS * ROW_PAIRS, KEY_PAIRS * ROW_PAIRS == 4 ? 2 : 1) void attn_bwd_k_kernel(DsqAttnBwdArgs a, int tiles, int splits)
{
    constexpr int HD = kRow<WIDTH>, STEPS = WIDTH / 16, DT = WIDTH / 32;
    typedef Tile<E, HD> T;
    typedef typename Operand<E>::type V8;
    constexpr int PAIRS = KEY_PAIRS * ROW_PAIRS, THREADS = 128 * PAIRS, KEYS = 32 * KEY_PAIRS, MINE = 32 * SUB, ROWS = MINE * ROW_PAIRS;
    // Tiles of queries (and of gradients, where 160 KB have room) go straight into a second buffer: 1 to 4 % of both backward kernels' time.
    constexpr bool DIRECT_Q = sizeof(E) == 2, DIRECT_G = sizeof(E) == 2 && WIDTH == 64;
    constexpr int TILE = ROWS * HD, TILES = 2 + DIRECT_Q + DIRECT_G, JOIN = (ROW_PAIRS - 1) * 2 * KEY_PAIRS * DT * 4096;
    __shared__ __align__(16) char room[most(TILES * TILE * (int)sizeof(E), JOIN)];
    __shared__ __align__(16) float handed[PAIRS][SUB][16 * 64], stats[2][ROWS];

    const int tid = threadIdx.x, lane = tid & 63, wave = wave_number(), r = lane & 31, h = lane >> 5;
    const int pair = wave % PAIRS, part = pair / KEY_PAIRS, group = a.q_heads / a.kv_heads;
    const bool values = wave < PAIRS;                            // sums dv, not dk
    // Workgroups go to the eight dies in turn: each die takes tiles side by side, which read the same rows.  (The first keys of a causal
    // prompt are seen by the most rows: they go first.)
    const int number = blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8, split = number / tiles % splits, kv = number / tiles / splits;
    if (kv >= a.kv_heads) return;
    const Sequence s = tile_of(a.q_starts, a.k_starts, a.q_rows, a.k_rows, a.sequences, true, KEYS, number % tiles);
    if (s.at < 0) return;

    const int first_key = s.at + pair % KEY_PAIRS * 32, key = first_key + r;
    const bool there = key < s.k_len;
    const int64_t token = s.k0 + key;
    const DsqHeads mine = values ? a.k : a.v;
    const E *its = (const E *)mine.p + token * mine.row + kv * mine.head;
    V8 own[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) own[i] = load_unit8(its, 2 * i + h, a.dim, there);
    // Row i sees keys up to i + off; rows from `first` on see one of the workgroup's, and rows from `all` on every one of the wave's.
    const int off = s.k_len - s.q_len;
    const int first = a.causal && s.at - off > 0 ? (s.at - off) / 32 * 32 : 0;
    const int all = a.causal ? first_key - off + 31 : 0;
    const float c = a.scale * kLog2e;

    Feed<E, HD, ROWS, DIRECT_Q, THREADS> qm;
    Feed<E, HD, ROWS, DIRECT_G, THREADS> gm;
    const auto q_tile = [&](int b) { return reinterpret_cast<E *>(room) + (DIRECT_Q ? b * TILE : 0); };
    const auto g_tile = [&](int b) { return reinterpret_cast<E *>(room) + (1 + DIRECT_Q + (DIRECT_G ? b : 0)) * TILE; };
    float stat = 0.0f;
    auto fetch = [&](int head, int at, int b) {
        qm.start(q_tile(b), (const E *)a.q.p + s.q0 * a.q.row + head * a.q.head, a.q.row, at, s.q_len, a.dim);
        gm.start(g_tile(b), (const E *)a.grad_out.p + s.q0 * a.grad_out.row + head * a.grad_out.head, a.grad_out.row, at, s.q_len, a.dim);
        if (tid < 2 * ROWS) {
            const int row = at + tid % ROWS;
            const float *numbers = (tid < ROWS ? a.lse : a.delta) + (int64_t)head * a.q_rows + s.q0;
            stat = row < s.q_len ? numbers[row] : 0.0f;
        }
    };
    v16f sum[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) sum[d] = zeros();
    // blocks of rows, head by head
    const int blocks = first < s.q_len ? (s.q_len - first + ROWS - 1) / ROWS : 0, from = (int)((int64_t)blocks * group * split / splits);
    const auto walk = [&](auto role) {
        constexpr bool VALUES = decltype(role)::value;
        int left = (int)((int64_t)blocks * group * (split + 1) / splits) - from;
        int head = blocks ? kv * group + from / blocks : 0, at = blocks ? first + from % blocks * ROWS : 0;
        if (left > 0) fetch(head, at, 0);
        v4f *const slot = reinterpret_cast<v4f *>(handed[pair][0]) + lane;
        for (int b = 0; left > 0; --left, b ^= 1) {
            E *const qt = q_tile(b), *const gt = g_tile(b);
            __syncthreads();
            qm.finish(qt);
            gm.finish(gt);
            if (tid < 2 * ROWS) stats[tid / ROWS][tid % ROWS] = tid < ROWS ? __builtin_fmaf(stat, kLog2e, -kLift<E>) : stat * kDrop<E>;
            __syncthreads();
            const int row0 = at + part * MINE;                      // the wave's first row
            at += ROWS;
            if (at >= s.q_len) at = first, ++head;
            if (left > 1) fetch(head, at, b ^ 1);
            v16f x[SUB];
            const E *rows = VALUES ? qt : gt;
#pragma unroll
            for (int u = 0; u < SUB; ++u) x[u] = zeros();
#pragma unroll
            for (int i = 0; i < STEPS; ++i)
#pragma unroll
                for (int u = 0; u < SUB; ++u) x[u] = multiply(T::row_operand(rows, part * MINE + u * 32 + r, i, h), own[i], x[u]);
            if (VALUES) {
#pragma unroll
                for (int u = 0; u < SUB; ++u) {
                    const int row = row0 + u * 32;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const v4f lse = *reinterpret_cast<const v4f *>(&stats[0][part * MINE + u * 32 + 8 * j + 4 * h]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[u][4 * j + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[u][4 * j + e], c, -lse[e]));
                    }
                    if (row < all || row + 32 > s.q_len) {
                        stay_a_branch();
                        // rows from `seeing` on, up to the last, see the lane's key
                        const int seeing = (a.causal ? key - off : 0) - row - 4 * h, last = s.q_len - row - 4 * h;
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[u][i] = ((8 * (i / 4) + i % 4 >= seeing) & (8 * (i / 4) + i % 4 < last)) ? x[u][i] : 0.0f;
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) slot[(u * 4 + j) * 64] = v4f{x[u][4 * j], x[u][4 * j + 1], x[u][4 * j + 2], x[u][4 * j + 3]};
                }
            }
            __syncthreads();
            if (!VALUES) {
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const v4f delta = *reinterpret_cast<const v4f *>(&stats[1][part * MINE + u * 32 + 8 * j + 4 * h]), p = slot[(u * 4 + j) * 64];
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[u][4 * j + e] = p[e] * __builtin_fmaf(x[u][4 * j + e], kDrop<E>, -delta[e]);
                    }
            }
            const E *columns = VALUES ? gt : qt;
#pragma unroll
            for (int u = 0; u < SUB; ++u)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const V8 w = operand_of<E>(x[u], half);
#pragma unroll
                    for (int d = 0; d < DT; ++d)
                        sum[d] = multiply(T::column_operand(columns, part * MINE + u * 32 + half * 16, d * 32, lane), w, sum[d]);
                }
        }
    };
    if (values) walk(std::true_type());
    else walk(std::false_type());
    join<DT>(sum, reinterpret_cast<float *>(room), wave / PAIRS * KEY_PAIRS + pair % KEY_PAIRS, 2 * KEY_PAIRS, part, ROW_PAIRS, lane);
    if (!there || part > 0) return;
    if (splits == 1) {
        const DsqHeadsOut out = values ? a.grad_v : a.grad_k;
        store_row<E, DT>((E *)out.p + token * out.row + kv * out.head, sum, values ? kDrop<E> : a.scale, h, a.dim);
    } else {
        store_row<float, DT>(a.partial + (((int64_t)split * 2 + (values ? 1 : 0)) * a.k_rows * a.kv_heads + token * a.kv_heads + kv) * a.dim, sum, 1.0f, h, a.dim);
    }
}

// The sums of the splits, four elements of a head a thread.
template <class E>
__global__ __launch_bounds__(256) void attn_bwd_join_kernel(DsqAttnBwdArgs a, int splits)
{
    const int64_t each = (int64_t)a.k_rows * a.kv_heads * a.dim, i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= each) return;
    const int d = (int)(i % a.dim), kv = (int)(i / a.dim % a.kv_heads), token = (int)(i / a.dim / a.kv_heads);
    if (a.k_starts && (token < a.k_starts[0] || token >= a.k_starts[a.sequences])) return;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < splits; ++s) sum += *reinterpret_cast<const v4f *>(a.partial + (2 * s + which) * each + i);
        const DsqHeadsOut out = which ? a.grad_v : a.grad_k;
        const float by = which ? kDrop<E> : a.scale;
        Side<E, 4> v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v.at[e] = (E)(sum[e] * by);
        store_side((E *)out.p + token * out.row + kv * out.head + d, v);
    }
}

template <class E, int WIDTH, int ROW_WAVES>
hipError_t queries(const DsqAttnBwdArgs &a, hipStream_t stream)
{
    const int tiles = attn_tiles(a.q_rows, 32 * ROW_WAVES, a.sequences, a.q_starts);
    attn_bwd_q_kernel<E, WIDTH, ROW_WAVES><<<(unsigned)((int64_t)attn_turns(tiles, a.sequences) * a.q_heads), 256, 0, stream>>>(a, tiles);
    return hipGetLastError();
}
template <class E, int WIDTH, int KEY_PAIRS, int ROW_PAIRS, int SUB>
hipError_t keys(const DsqAttnBwdArgs &a, hipStream_t stream)
{
    const int tiles = attn_tiles(a.k_rows, 32 * KEY_PAIRS, a.sequences, a.q_starts);
    const int64_t groups = (int64_t)tiles * a.kv_heads, each = (int64_t)a.k_rows * a.kv_heads * a.dim;
    // Workgroups for two rounds of the card, as far as there are rows and room.
    int64_t splits = 512 / groups;
    const int64_t blocks = (a.q_rows / (32 * SUB * ROW_PAIRS) + 1LL) * (a.q_heads / a.kv_heads), room = (int64_t)(a.partial_bytes / 8) / each;
    for (const int64_t limit : {blocks, room, (int64_t)16}) splits = splits < limit ? splits : limit;
    splits = splits < 1 ? 1 : splits;
    attn_bwd_k_kernel<E, WIDTH, KEY_PAIRS, ROW_PAIRS, SUB>
        <<<(unsigned)((groups * splits + 7) / 8 * 8), 128 * KEY_PAIRS * ROW_PAIRS, 0, stream>>>(a, tiles, (int)splits);
    if (const hipError_t e = hipGetLastError()) return e;
    if (splits > 1) attn_bwd_join_kernel<E><<<(unsigned)((each / 4 + 255) / 256), 256, 0, stream>>>(a, (int)splits);
    return hipGetLastError();
}

template <class E, int WIDTH>
hipError_t launch(const DsqAttnBwdArgs &a, hipStream_t stream)
{
    constexpr bool SINGLE = sizeof(E) == 4;
    if (a.q_rows > 0) {
        const bool few = attn_bwd_rows(sizeof(E), WIDTH, a.q_rows, a.q_heads) == 32;
        if (const hipError_t e = few ? queries<E, WIDTH, 1>(a, stream) : queries<E, WIDTH, SINGLE ? 2 : 4>(a, stream)) return e;
    }
    return a.k_rows > 0 ? keys<E, WIDTH, SINGLE ? 1 : 2, 2, 2>(a, stream) : hipSuccess;
}

template <class E>
hipError_t of_dim(const DsqAttnBwdArgs &a, hipStream_t stream)
{
    switch (attn_width(a.dim)) {
    case 64: return launch<E, 64>(a, stream);
    case 96: return launch<E, 96>(a, stream);
    default: return launch<E, 128>(a, stream);
    }
}

}  // namespace

// Eight times a binary32 dk and dv of as many keys as there are rows, at most 32 MB: 512 workgroups' worth.
size_t dsq_attn_bwd_partial_bytes(int q_rows, int q_heads)
{
    const size_t all = (size_t)q_rows * q_heads * 8192;
    return all < (32u << 20) ? all : 32u << 20;
}

hipError_t dsq_launch_attention_bwd(const DsqAttnBwdArgs &a, int type, hipStream_t stream)
{
    if (type == DSQ_T_F32) return of_dim<float>(a, stream);
    if (type == DSQ_T_F16) return of_dim<_Float16>(a, stream);
    return of_dim<__bf16>(a, stream);
}
