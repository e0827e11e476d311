// Attention over whole prompts, backward.
//
//   p_ij = exp(s_ij - lse_i),  D_i = do_i . o_i,  ds_ij = p_ij (do_i . v_j - D_i)
//   dv_j = sum_i p_ij do_i,  dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i
//
// Two kernels, each of which forms the scores again, so that every sum has one owner and no atomics are needed: the same bits every
// time.  One owns rows of queries (D and dq), the other keys, over all heads that share them (dk and dv).  In both a
// lane holds a column of the 32x32 results, so probabilities and ds are the second operand of the next product as they lie
// in registers (attn_device.h).
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

__device__ __forceinline__ v16f zeros()
{
    v16f z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.0f;
    return z;
}

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

template <class E, int HD, int ROWS>
struct Mover {
    typedef Tile<E, HD> T;
    static constexpr int PIECES = ROWS * HD * (int)sizeof(E) / 16 / 256;     // 16-byte pieces of a tile a thread moves
    v4u at[PIECES];
    // rows first .. first + ROWS - 1 of `p`, zeros from `end` on
    __device__ __forceinline__ void fetch(const E *p, int64_t stride, int first, int end, int dim)
    {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int piece = threadIdx.x + 256 * i, j = first + piece / T::UNITS, u = piece % T::UNITS;
            at[i] = j < end && u * T::PER < dim ? *reinterpret_cast<const v4u *>(p + j * stride + u * T::PER) : v4u{0, 0, 0, 0};
        }
    }
    __device__ __forceinline__ void put(E *t) const
    {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int piece = threadIdx.x + 256 * i;
            *reinterpret_cast<v4u *>(t + T::place(piece / T::UNITS, piece % T::UNITS)) = at[i];
        }
    }
};

// ---- queries ------------------------------------------------------------------------------------

template <class E, int HD>
__global__ __launch_bounds__(256, sizeof(E) == 2 || HD == 64 ? 2 : 1) void attn_bwd_q_kernel(DsqAttnBwdArgs a, int tiles)
{
    typedef Tile<E, HD> T;
    typedef typename Operand<E>::type V8;
    constexpr int ROWS = 128, KEYS = 32, STEPS = HD / 16, DT = HD / 32;
    __shared__ __align__(16) E ks[2][KEYS * HD], vs[2][KEYS * HD];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 31, h = lane >> 5;
    const int of = blockIdx.x / a.q_heads, turn = blockIdx.x % a.q_heads;
    const int head = a.q_heads % 8 == 0 ? turn % 8 * (a.q_heads / 8) + turn / 8 : turn;
    const int kv = head / (a.q_heads / a.kv_heads);
    const Sequence s = tile_of(a.q_starts, a.k_starts, a.q_rows, a.k_rows, a.sequences, false, ROWS, tiles - 1 - of);
    if (s.at < 0) return;

    const E *kp = (const E *)a.k.p + s.k0 * a.k.row + kv * a.k.head, *vp = (const E *)a.v.p + s.k0 * a.v.row + kv * a.v.head;
    const int last = s.at + ROWS < s.q_len ? s.at + ROWS - 1 : s.q_len - 1;
    const int k_end = visible(s, a.causal, last), count = (k_end + KEYS - 1) / KEYS;

    const int row = s.at + wave * 32 + r;
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
    if (there && h == 0) a.delta[stat] = delta;
    const int seen = there ? visible(s, a.causal, row) : 0;
    const float lse = seen > 0 ? a.lse[stat] * kLog2e - kLift<E> : 0.0f;
    delta *= kDrop<E>;
    const int first_row = s.at + wave * 32, last_row = first_row + 31 < s.q_len ? first_row + 31 : s.q_len - 1;
    const int whole = first_row + 31 < s.q_len ? visible(s, a.causal, first_row) : 0;
    const int any = first_row < s.q_len ? visible(s, a.causal, last_row) : 0;
    const float c = a.scale * kLog2e;

    Mover<E, HD, KEYS> km, vm;
    v16f dq[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) dq[d] = zeros();
    if (count > 0) {
        km.fetch(kp, a.k.row, 0, k_end, a.dim);
        vm.fetch(vp, a.v.row, 0, k_end, a.dim);
        km.put(ks[0]);
        vm.put(vs[0]);
        __syncthreads();
    }
    for (int t = 0; t < count; ++t) {
        const E *kt = ks[t & 1], *vt = vs[t & 1];
        if (t + 1 < count) {
            km.fetch(kp, a.k.row, (t + 1) * KEYS, k_end, a.dim);
            vm.fetch(vp, a.v.row, (t + 1) * KEYS, k_end, a.dim);
        }
        if (t * KEYS < any) {
            v16f x = zeros(), y = zeros();
#pragma unroll
            for (int i = 0; i < STEPS; ++i) x = multiply(T::row_operand(kt, r, i, h), q[i], x);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) y = multiply(T::row_operand(vt, r, i, h), g[i], y);
            const bool masked = (t + 1) * KEYS > whole;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], c, -lse));
                x[i] = p * __builtin_fmaf(y[i], kDrop<E>, -delta);
            }
            if (masked) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = t * KEYS + 8 * (i / 4) + 4 * h + i % 4 < seen ? x[i] : 0.0f;
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const V8 ds = operand_of<E>(x, half);
#pragma unroll
                for (int d = 0; d < DT; ++d) dq[d] = multiply(T::column_operand(kt, half * 16, d * 32, lane), ds, dq[d]);
            }
        }
        if (t + 1 < count) {
            km.put(ks[(t + 1) & 1]);
            vm.put(vs[(t + 1) & 1]);
        }
        __syncthreads();
    }
    if (there) store_row<E, DT>((E *)a.grad_q.p + token * a.grad_q.row + head * a.grad_q.head, dq, a.scale, h, a.dim);
}

// ---- keys and values ------------------------------------------------------------------------------

template <class E, int HD>
__global__ __launch_bounds__(256, 1) void attn_bwd_k_kernel(DsqAttnBwdArgs a, int tiles)
{
    typedef Tile<E, HD> T;
    typedef typename Operand<E>::type V8;
    constexpr int KEYS = 128, ROWS = 32, STEPS = HD / 16, DT = HD / 32;
    __shared__ __align__(16) E qs[2][ROWS * HD], gs[2][ROWS * HD];
    __shared__ __align__(16) float stats[2][2][ROWS];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 31, h = lane >> 5;
    const int of = blockIdx.x / a.kv_heads, kv = blockIdx.x % a.kv_heads, group = a.q_heads / a.kv_heads;
    // (the first keys of a causal prompt are seen by the most rows: they go first)
    const Sequence s = tile_of(a.q_starts, a.k_starts, a.q_rows, a.k_rows, a.sequences, true, KEYS, of);
    if (s.at < 0) return;

    const int key = s.at + wave * 32 + r;
    const bool there = key < s.k_len;
    const int64_t token = s.k0 + key;
    const E *kp = (const E *)a.k.p + token * a.k.row + kv * a.k.head, *vp = (const E *)a.v.p + token * a.v.row + kv * a.v.head;
    V8 k[STEPS], v[STEPS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        k[i] = load_unit8(kp, 2 * i + h, a.dim, there);
        v[i] = load_unit8(vp, 2 * i + h, a.dim, there);
    }
    // Row i sees keys up to i + off; rows from `first` on see one of the workgroup's, rows from `all` on every one of the wave's.
    const int off = s.k_len - s.q_len;
    const int first = a.causal && s.at - off > 0 ? s.at - off : 0, t0 = first / ROWS;
    const int count = s.q_len > t0 * ROWS ? (s.q_len + ROWS - 1) / ROWS - t0 : 0, turns = count * group;
    const int wave_first = a.causal ? s.at + wave * 32 - off : 0, all = a.causal ? wave_first + 31 : 0;
    const float c = a.scale * kLog2e;

    Mover<E, HD, ROWS> qm, gm;
    float stat = 0.0f;
    auto fetch = [&](int n) {
        const int head = kv * group + n / count, at = (t0 + n % count) * ROWS;
        qm.fetch((const E *)a.q.p + s.q0 * a.q.row + head * a.q.head, a.q.row, at, s.q_len, a.dim);
        gm.fetch((const E *)a.grad_out.p + s.q0 * a.grad_out.row + head * a.grad_out.head, a.grad_out.row, at, s.q_len, a.dim);
        if (tid < 2 * ROWS) {
            const int row = at + tid % ROWS;
            const int64_t i = (int64_t)head * a.q_rows + s.q0 + row;
            // (rows that are not there see nothing)
            if (tid < ROWS) stat = row < s.q_len ? a.lse[i] * kLog2e - kLift<E> : 0.0f;
            else stat = row < s.q_len ? a.delta[i] * kDrop<E> : 0.0f;
        }
    };
    auto put = [&](int b) {
        qm.put(qs[b]);
        gm.put(gs[b]);
        if (tid < 2 * ROWS) stats[b][tid / ROWS][tid % ROWS] = stat;
    };

    v16f dk[DT], dv[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) dk[d] = zeros(), dv[d] = zeros();
    if (turns > 0) {
        fetch(0);
        put(0);
        __syncthreads();
    }
    for (int n = 0; n < turns; ++n) {
        const E *qt = qs[n & 1], *gt = gs[n & 1];
        const int at = (t0 + n % count) * ROWS;
        if (n + 1 < turns) fetch(n + 1);
        if (at + ROWS > wave_first) {
            v16f x = zeros(), y = zeros();
#pragma unroll
            for (int i = 0; i < STEPS; ++i) x = multiply(T::row_operand(qt, r, i, h), k[i], x);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) y = multiply(T::row_operand(gt, r, i, h), v[i], y);
            const bool masked = at < all || at + ROWS > s.q_len;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const v4f lse = *reinterpret_cast<const v4f *>(&stats[n & 1][0][8 * j + 4 * h]);
                const v4f delta = *reinterpret_cast<const v4f *>(&stats[n & 1][1][8 * j + 4 * h]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = 4 * j + e, row = at + 8 * j + 4 * h + e;
                    float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], c, -lse[e]));
                    float ds = p * __builtin_fmaf(y[i], kDrop<E>, -delta[e]);
                    if (masked) {
                        const bool sees = row < s.q_len && (!a.causal || key <= row + off);
                        p = sees ? p : 0.0f;
                        ds = sees ? ds : 0.0f;
                    }
                    x[i] = p;
                    y[i] = ds;
                }
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const V8 p = operand_of<E>(x, half), ds = operand_of<E>(y, half);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    dv[d] = multiply(T::column_operand(gt, half * 16, d * 32, lane), p, dv[d]);
                    dk[d] = multiply(T::column_operand(qt, half * 16, d * 32, lane), ds, dk[d]);
                }
            }
        }
        if (n + 1 < turns) put((n + 1) & 1);
        __syncthreads();
    }
    if (there) {
        store_row<E, DT>((E *)a.grad_k.p + token * a.grad_k.row + kv * a.grad_k.head, dk, a.scale, h, a.dim);
        store_row<E, DT>((E *)a.grad_v.p + token * a.grad_v.row + kv * a.grad_v.head, dv, kDrop<E>, h, a.dim);
    }
}

template <class E, int HD>
hipError_t launch(const DsqAttnBwdArgs &a, hipStream_t stream)
{
    const auto tiles = [&](int rows) { return a.q_starts ? rows / 128 + a.sequences : (rows + 127) / 128; };
    const int tq = tiles(a.q_rows), tk = tiles(a.k_rows);
    if (a.q_rows > 0) {
        attn_bwd_q_kernel<E, HD><<<(unsigned)((int64_t)tq * a.q_heads), 256, 0, stream>>>(a, tq);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    if (a.k_rows > 0) attn_bwd_k_kernel<E, HD><<<(unsigned)((int64_t)tk * a.kv_heads), 256, 0, stream>>>(a, tk);
    return hipGetLastError();
}

template <class E>
hipError_t of_dim(const DsqAttnBwdArgs &a, hipStream_t stream)
{
    return a.dim <= 64 ? launch<E, 64>(a, stream) : launch<E, 128>(a, stream);
}

}  // namespace

hipError_t dsq_launch_attention_bwd(const DsqAttnBwdArgs &a, int type, hipStream_t stream)
{
    if (type == DSQ_T_F32) return of_dim<float>(a, stream);
    if (type == DSQ_T_F16) return of_dim<_Float16>(a, stream);
    return of_dim<__bf16>(a, stream);
}
