// Attention over whole prompts, packed one behind the other, forward.
//
//   o_i = sum over visible j of p_ij v_j,  p_ij = exp(s_ij - m_i) / l_i,  s_ij = scale q_i . k_j
//
// One pass over the keys with the running maximum and sum of the softmax.  A workgroup of four waves owns 128 rows of one head, a
// wave 32 of them; tiles of keys and values go through LDS, the next tile's loads under way.  Scores are formed transposed, K Q^T,
// so that a lane holds one row's scores: maximum, sum and the factor of a raised maximum need no exchange but one between the two
// lanes of a row, and the probabilities are the second operand of V^T P^T as they lie in registers (attn_device.h).
#include "attn_device.h"

namespace {

template <class E, int HD>
struct Fwd {
    static constexpr int ROWS = 128, KEYS = sizeof(E) == 2 ? 64 : 32;
    static constexpr int STEPS = HD / 16, DT = HD / 32, KT = KEYS / 32;
    static constexpr int PIECES = KEYS * HD * (int)sizeof(E) / 16 / 256;     // 16-byte pieces of a tile a thread moves
    typedef Tile<E, HD> T;
};

// Keys of one row of a packed prompt.
template <class E>
struct PromptKeys {
    const E *k, *v;
    int64_t k_row, v_row;
    int n;
    __device__ int count() const { return n; }
    __device__ bool seen(int) const { return true; }
    __device__ const E *key(int j) const { return k + j * k_row; }
    __device__ const E *value(int j) const { return v + j * v_row; }
};

template <class E, int HD>
__global__ __launch_bounds__(256, sizeof(E) == 2 || HD == 64 ? 2 : 1) void attn_fwd_kernel(DsqAttnArgs a, int tiles)
{
    typedef Fwd<E, HD> F;
    typedef typename F::T T;
    typedef typename Operand<E>::type V8;
    __shared__ __align__(16) E ks[2][F::KEYS * HD], vs[2][F::KEYS * HD];

    // heads that share keys meet on one of the eight dies, which take workgroups in turn
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 31, h = lane >> 5;
    const int of = blockIdx.x / a.q_heads, turn = blockIdx.x % a.q_heads;
    const int head = a.q_heads % 8 == 0 ? turn % 8 * (a.q_heads / 8) + turn / 8 : turn;
    const int kv = head / (a.q_heads / a.kv_heads);
    // (the last tiles of a causal prompt are the longest: they go first)
    const Sequence s = tile_of(a.q_starts, a.k_starts, a.q_rows, a.k_rows, a.sequences, false, F::ROWS, tiles - 1 - of);
    if (s.at < 0) return;

    const E *kp = (const E *)a.k.p + s.k0 * a.k.row + kv * a.k.head, *vp = (const E *)a.v.p + s.k0 * a.v.row + kv * a.v.head;
    const int last = s.at + F::ROWS < s.q_len ? s.at + F::ROWS - 1 : s.q_len - 1;
    const int k_end = visible(s, a.causal, last), count = (k_end + F::KEYS - 1) / F::KEYS;

    const int row = s.at + wave * 32 + r;                    // this lane's row
    const bool there = row < s.q_len;
    const E *qp = (const E *)a.q.p + (int64_t)(s.q0 + row) * a.q.row + head * a.q.head;
    V8 q[F::STEPS];
#pragma unroll
    for (int i = 0; i < F::STEPS; ++i) q[i] = load_unit8(qp, 2 * i + h, a.dim, there);
    const int seen = there ? visible(s, a.causal, row) : 0;
    // keys that all of the wave's rows see, and that any does
    const int first_row = s.at + wave * 32, last_row = first_row + 31 < s.q_len ? first_row + 31 : s.q_len - 1;
    const int whole = first_row + 31 < s.q_len ? visible(s, a.causal, first_row) : 0;
    const int any = first_row < s.q_len ? visible(s, a.causal, last_row) : 0;

    v4u kr[F::PIECES], vr[F::PIECES];
    auto fetch = [&](int t) {
#pragma unroll
        for (int i = 0; i < F::PIECES; ++i) {
            const int piece = tid + 256 * i, j = t * F::KEYS + piece / T::UNITS, u = piece % T::UNITS;
            const bool ok = j < k_end && u * T::PER < a.dim;
            kr[i] = ok ? *reinterpret_cast<const v4u *>(kp + j * a.k.row + u * T::PER) : v4u{0, 0, 0, 0};
            vr[i] = ok ? *reinterpret_cast<const v4u *>(vp + j * a.v.row + u * T::PER) : v4u{0, 0, 0, 0};
        }
    };
    auto put = [&](int b) {
#pragma unroll
        for (int i = 0; i < F::PIECES; ++i) {
            const int piece = tid + 256 * i, at = T::place(piece / T::UNITS, piece % T::UNITS);
            *reinterpret_cast<v4u *>(ks[b] + at) = kr[i];
            *reinterpret_cast<v4u *>(vs[b] + at) = vr[i];
        }
    };

    const float c = a.scale * kLog2e;
    float m = kNoKey, l = 0.0f;
    v16f o[F::DT];
#pragma unroll
    for (int d = 0; d < F::DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;

    if (count > 0) {
        fetch(0);
        put(0);
        __syncthreads();
    }
    for (int t = 0; t < count; ++t) {
        const E *kt = ks[t & 1], *vt = vs[t & 1];
        if (t + 1 < count) fetch(t + 1);
        if (t * F::KEYS < any) {
            v16f x[F::KT];
#pragma unroll
            for (int n = 0; n < F::KT; ++n) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[n][i] = 0.0f;
#pragma unroll
                for (int i = 0; i < F::STEPS; ++i) x[n] = multiply(T::row_operand(kt, n * 32 + r, i, h), q[i], x[n]);
            }
            if ((t + 1) * F::KEYS > whole) {
#pragma unroll
                for (int n = 0; n < F::KT; ++n)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        x[n][i] = t * F::KEYS + n * 32 + 8 * (i / 4) + 4 * h + i % 4 < seen ? x[n][i] : -INFINITY;
            }
            float most = x[0][0];
#pragma unroll
            for (int n = 0; n < F::KT; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) most = __builtin_elementwise_maximum(most, x[n][i]);
            most = both_max(most) * c;
            // The reference is raised only where a score passes it by 2^8: up to there sums and operands lose nothing.
            if (__any(most > m + 8.0f)) {
                const float next = most > m ? most : m, f = __builtin_amdgcn_exp2f(m - next);
                m = next;
                l *= f;
#pragma unroll
                for (int d = 0; d < F::DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= f;
            }
#pragma unroll
            for (int n = 0; n < F::KT; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    x[n][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[n][i], c, -m));
                    l += x[n][i];
                }
#pragma unroll
            for (int n = 0; n < F::KT; ++n)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const V8 p = operand_of<E>(x[n], half);
#pragma unroll
                    for (int d = 0; d < F::DT; ++d)
                        o[d] = multiply(T::column_operand(vt, n * 32 + half * 16, d * 32, lane), p, o[d]);
                }
        }
        if (t + 1 < count) put((t + 1) & 1);
        __syncthreads();
    }

    l = both_sum(l);
    const float inv = seen > 0 ? 1.0f / l : 0.0f;
    bool bad = false;
    E *op = (E *)a.out.p + (int64_t)(s.q0 + row) * a.out.row + head * a.out.head;
#pragma unroll
    for (int d = 0; d < F::DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            Side<E, 4> v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float y = seen > 0 ? o[d][4 * i + e] * inv : 0.0f;
                bad |= !is_finite(y);
                v.at[e] = (E)y;
            }
            const int at = d * 32 + 8 * i + 4 * h;
            if (there && at < a.dim) store_side(op + at, v);
        }
    if (a.lse && there && h == 0) a.lse[(int64_t)head * a.q_rows + s.q0 + row] = seen > 0 ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;

    uint64_t again = __ballot(bad && there);
    again = (again | again >> 32) & 0xffffffffu;
    while (again) {
        const int i = __ffsll((unsigned long long)again) - 1, at = first_row + i;
        again &= again - 1;
        const PromptKeys<E> keys = {kp, vp, a.k.row, a.v.row, visible(s, a.causal, at)};
        float y[2];
        const float log2 = row_again<E>((const E *)a.q.p + (int64_t)(s.q0 + at) * a.q.row + head * a.q.head, a.dim, c, keys, y);
        E *to = (E *)a.out.p + (int64_t)(s.q0 + at) * a.out.row + head * a.out.head;
        if (lane < a.dim) to[lane] = (E)y[0];
        if (lane + 64 < a.dim) to[lane + 64] = (E)y[1];
        if (a.lse && lane == 0) a.lse[(int64_t)head * a.q_rows + s.q0 + at] = log2 * kLn2;
    }
}

template <class E, int HD>
hipError_t launch(const DsqAttnArgs &a, hipStream_t stream)
{
    const int tiles = a.q_starts ? a.q_rows / Fwd<E, HD>::ROWS + a.sequences : (a.q_rows + Fwd<E, HD>::ROWS - 1) / Fwd<E, HD>::ROWS;
    attn_fwd_kernel<E, HD><<<(unsigned)((int64_t)tiles * a.q_heads), 256, 0, stream>>>(a, tiles);
    return hipGetLastError();
}

template <class E>
hipError_t of_dim(const DsqAttnArgs &a, hipStream_t stream)
{
    return a.dim <= 64 ? launch<E, 64>(a, stream) : launch<E, 128>(a, stream);
}

}  // namespace

hipError_t dsq_launch_attention(const DsqAttnArgs &a, int type, hipStream_t stream)
{
    if (type == DSQ_T_F32) return of_dim<float>(a, stream);
    if (type == DSQ_T_F16) return of_dim<_Float16>(a, stream);
    return of_dim<__bf16>(a, stream);
}
