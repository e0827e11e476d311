// Norms of queries and keys for each head with the rotation by their positions in the same pass, forward and backward.
//
//   n = x r w, r = 1 / sqrt(mean of x^2 + eps);  pair j = (a, b), t = position[axis j] * frequency[j]:
//   a' = a cos t - b sin t, b' = b cos t + a sin t
//   backward: (ga, gb) = (ga' cos t + gb' sin t, gb' cos t - ga' sin t), u = g w, m = x r:  gx = r (u - m mean(u m)), gw = sum of g m
//
// A lane holds both elements of eight pairs, 16 of a head's elements in two units of eight: pairs of halves are the units c and
// rope_dim / 16 + c, neighbouring pairs, and the elements behind the rotated ones, the units 2c and 2c + 1.  Angles are
// formed once a row and workgroup, the product and its remainder in binary64: a position of 2^31 still has its angle to 2^-20.
// Bound by HBM bandwidth, and by latency for a few rows.  Measured: bfloat16, 4096 rows, 32 + 8 heads of 128 and a cache, 101 MB,
// 25.5 us (4.0 TB/s; a row's 256 bytes of a cached head go to a place of their own: 21.3 with neighbouring slots); 8 rows 4.2 us;
// binary32, 80 elements, both passes 128 MB, 45 us (five of eight lanes are busy).  Backward, 4096 rows, 32 + 8 heads of 128: bfloat16 and
// float16 43 us (2.9 TB/s), binary32 59 (4.3).
#include "attn_device.h"

namespace {

constexpr int kThreads = 256;                // the most of a workgroup
constexpr int kRows = 8;                     // the most rows of a workgroup

// What a workgroup takes: all heads of `rows` rows, or `heads` of one.
struct Share {
    int rows, heads, blocks, threads;
};

// What a lane holds: which head of which of the workgroup's rows, and which units of it.
struct Place {
    int row, unit, c, a, b;                  // unit: q heads, k heads, v heads; c: lane of the head; a, b: units of eight elements, or -1
    bool turns;
};

template <int LANES>
__device__ __forceinline__ Place place_of(const Share &share, int dim, int pairs, int interleaved)
{
    Place p;
    const int item = threadIdx.x / LANES;
    p.row = item / share.heads;
    p.unit = p.row < share.rows ? blockIdx.y * share.heads + item % share.heads : 1 << 30;
    if (p.row >= share.rows) p.row = 0;      // (lanes past the last row have nothing to do)
    p.c = threadIdx.x % LANES;
    const int turning = pairs / 8;
    p.turns = p.c < turning;
    const bool halves = p.turns && !interleaved;
    p.a = halves ? p.c : 2 * p.c;
    p.b = halves ? turning + p.c : 2 * p.c + 1;
    if (p.a >= dim / 8) p.a = -1;
    if (p.b >= dim / 8) p.b = -1;
    return p;
}

template <class E>
__device__ __forceinline__ void load16(const E *head, const Place &p, int dim, typename Operand<E>::type &lo, typename Operand<E>::type &hi)
{
    lo = load_unit8(head, p.a, dim, p.a >= 0);
    hi = load_unit8(head, p.b, dim, p.b >= 0);
}
template <class E>
__device__ __forceinline__ void store8(E *to, const typename Operand<E>::type &v)
{
    if constexpr (sizeof(E) == 2) {
        *reinterpret_cast<typename Operand<E>::type *>(to) = v;
    } else {
        *reinterpret_cast<v4f *>(to) = __builtin_shufflevector(v, v, 0, 1, 2, 3);
        *reinterpret_cast<v4f *>(to + 4) = __builtin_shufflevector(v, v, 4, 5, 6, 7);
    }
}

template <int LANES>
__device__ __forceinline__ float lanes_sum(float v)
{
#pragma unroll
    for (int off = LANES / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}
template <int LANES>
__device__ __forceinline__ double lanes_sum(double v)
{
#pragma unroll
    for (int off = LANES / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// 1 / rms of 16 elements a lane; squares in binary64, so nothing over- or underflows.  0 for a head with an infinity (the step that makes
// the reciprocal root exact would be infinity times zero): its finite elements are normed to 0.
template <int LANES>
__device__ __forceinline__ float rms_of(const float *x, int dim, float eps)
{
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < 16; ++i) s = __builtin_fma((double)x[i], (double)x[i], s);
    const double mean = lanes_sum<LANES>(s) / dim + (double)eps;
    const double y = __builtin_amdgcn_rsq(mean);
    return y == 0.0 ? 0.0f : (float)(y * __builtin_fma(-0.5 * mean * y, y, 1.5));
}

// Cosine and sine of the pairs of `count` rows from `row` on, 256 numbers a row.
__device__ __forceinline__ void angles(float *table, const int32_t *positions, const uint8_t *pair_axis, const float *frequencies, int rows, int axes,
                                       int pairs, int row, int count)
{
    for (int i = threadIdx.x; i < pairs * count; i += blockDim.x) {
        const int r = count == 1 ? 0 : i / pairs, j = i - r * pairs;
        if (row + r >= rows) return;
        int axis = pair_axis ? pair_axis[j] : 0;
        axis = axis < axes ? axis : axes - 1;
        const double turns = (double)positions[(int64_t)axis * rows + row + r] * (double)frequencies[j] * 0.31830988618379067154;
        float s, c;
        sincospif((float)(turns - 2.0 * rint(0.5 * turns)), &s, &c);
        table[r * 256 + 2 * j] = c;
        table[r * 256 + 2 * j + 1] = s;
    }
}

// Pairs in order: x[0 .. 7] and x[8 .. 15] are their first and second elements.
__device__ __forceinline__ void to_pairs(float *x, bool neighbours)
{
    if (!neighbours) return;
    float y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = x[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = y[2 * i], x[i + 8] = y[2 * i + 1];
}
__device__ __forceinline__ void from_pairs(float *x, bool neighbours)
{
    if (!neighbours) return;
    float y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = x[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[2 * i] = y[i], x[2 * i + 1] = y[i + 8];
}

// by: 1 forward, -1 back
__device__ __forceinline__ void turn(float *x, const float *table, const Place &p, int interleaved, float by)
{
    if (!p.turns) return;
    to_pairs(x, interleaved);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float c = table[2 * (8 * p.c + i)], s = by * table[2 * (8 * p.c + i) + 1];
        const float a = x[i], b = x[i + 8];
        x[i] = __builtin_fmaf(a, c, -b * s);
        x[i + 8] = __builtin_fmaf(b, c, a * s);
    }
    from_pairs(x, interleaved);
}

template <class E, int LANES>
__global__ __launch_bounds__(kThreads) void head_rope_kernel(DsqRopeArgs a, Share share)
{
    typedef typename Operand<E>::type V8;
    __shared__ __align__(16) float table[kRows * 256];
    const int row0 = blockIdx.x * share.rows, units = a.q_heads + a.kv_heads + (a.cache.k ? a.kv_heads : 0);
    const Place p = place_of<LANES>(share, a.dim, a.pairs, a.interleaved);
    const int row = row0 + p.row;
    const bool there = p.unit < units && row < a.rows, is_q = p.unit < a.q_heads, is_v = p.unit >= a.q_heads + a.kv_heads;
    const int head = is_q ? p.unit : is_v ? p.unit - a.q_heads - a.kv_heads : p.unit - a.q_heads;
    const DsqHeads in = is_q ? a.q : is_v ? a.v : a.k;
    V8 lo = {}, hi = {};
    int64_t slot = -1;
    if (there) {
        load16((const E *)in.p + row * in.row + head * in.head, p, a.dim, lo, hi);
        if (a.cache.k && !is_q) slot = a.cache.slots[row];
    }
    angles(table, a.positions, a.pair_axis, a.frequencies, a.rows, a.axes, a.pairs, row0, share.rows);
    __syncthreads();
    if (!there) return;
    if (!is_v) {
        float x[16];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)lo[i], x[i + 8] = (float)hi[i];
        if (a.eps > 0.0f) {
            const float r = rms_of<LANES>(x, a.dim, a.eps);
            const E *weight = (const E *)(is_q ? a.q_weight : a.k_weight);
            V8 wl, wh;
            if (weight) load16(weight, p, a.dim, wl, wh);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] = x[i] * r * (weight ? (float)wl[i] : 1.0f);
                x[i + 8] = x[i + 8] * r * (weight ? (float)wh[i] : 1.0f);
            }
        }
        turn(x, table + p.row * 256, p, a.interleaved, 1.0f);
#pragma unroll
        for (int i = 0; i < 8; ++i) lo[i] = (E)x[i], hi[i] = (E)x[i + 8];
        const DsqHeadsOut out = is_q ? a.q_out : a.k_out;
        if (out.p) {
            E *to = (E *)out.p + row * out.row + head * out.head;
            if (p.a >= 0) store8(to + 8 * p.a, lo);
            if (p.b >= 0) store8(to + 8 * p.b, hi);
        }
    }
    const int64_t page = slot >> a.cache.page_bits;
    if (slot >= 0 && page < a.cache.pages) {
        E *to = (E *)(is_v ? a.cache.v : a.cache.k) + (((page * a.kv_heads + head) << a.cache.page_bits) + (slot & ((1 << a.cache.page_bits) - 1))) * a.dim;
        if (p.a >= 0) store8(to + 8 * p.a, lo);
        if (p.b >= 0) store8(to + 8 * p.b, hi);
    }
}

// A workgroup takes its rows in turn, the next ones' heads and angles under way, and keeps the weights' gradients of its heads in registers.
template <class E, int LANES>
__global__ __launch_bounds__(kThreads) void head_rope_bwd_kernel(DsqRopeBwdArgs a, Share share)
{
    typedef typename Operand<E>::type V8;
    constexpr int WIDE = LANES * 16;
    __shared__ __align__(16) float table[2][kRows * 256];
    __shared__ float sums[kThreads * 16];
    const int units = a.q_heads + a.kv_heads;
    const Place p = place_of<LANES>(share, a.dim, a.pairs, a.interleaved);
    const bool mine = p.unit < units, is_q = p.unit < a.q_heads;
    const int head = is_q ? p.unit : p.unit - a.q_heads;
    const DsqHeads in = is_q ? a.q : a.k, grad = is_q ? a.grad_q_out : a.grad_k_out;
    const DsqHeadsOut out = is_q ? a.grad_q : a.grad_k;
    const E *weight = (const E *)(is_q ? a.q_weight : a.k_weight);
    V8 wl, wh;
#pragma unroll
    for (int i = 0; i < 8; ++i) wl[i] = wh[i] = (E)1.0f;
    if (weight) load16(weight, p, a.dim, wl, wh);
    float gw[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) gw[i] = 0.0f;

    V8 xl = {}, xh = {}, gl = {}, gh = {};
    auto fetch = [&](int row) {
        if (mine && row < a.rows) {
            load16((const E *)grad.p + row * grad.row + head * grad.head, p, a.dim, gl, gh);
            if (a.eps > 0.0f) load16((const E *)in.p + row * in.row + head * in.head, p, a.dim, xl, xh);
        }
    };
    const int step = gridDim.x * share.rows;
    int b = 0, row0 = blockIdx.x * share.rows;
    fetch(row0 + p.row);
    angles(table[0], a.positions, a.pair_axis, a.frequencies, a.rows, a.axes, a.pairs, row0, share.rows);
    for (; row0 < a.rows; row0 += step, b ^= 1) {
        const int row = row0 + p.row;
        const bool there = mine && row < a.rows;
        float g[16], x[16];
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = (float)gl[i], g[i + 8] = (float)gh[i], x[i] = (float)xl[i], x[i + 8] = (float)xh[i];
        __syncthreads();
        if (row0 + step < a.rows) {
            fetch(row + step);
            angles(table[b ^ 1], a.positions, a.pair_axis, a.frequencies, a.rows, a.axes, a.pairs, row0 + step, share.rows);
        }
        turn(g, table[b] + p.row * 256, p, a.interleaved, -1.0f);
        if (a.eps > 0.0f) {
            float dot = 0.0f;
            const float r = rms_of<LANES>(x, a.dim, a.eps);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[i] *= r;
                if (there) gw[i] = __builtin_fmaf(g[i], x[i], gw[i]);
                g[i] *= (float)(i < 8 ? wl[i % 8] : wh[i % 8]);
                dot = __builtin_fmaf(g[i], x[i], dot);
            }
            dot = lanes_sum<LANES>(dot) / a.dim;
#pragma unroll
            for (int i = 0; i < 16; ++i) g[i] = r * __builtin_fmaf(-x[i], dot, g[i]);
        }
        if (there) {
            V8 lo, hi;
#pragma unroll
            for (int i = 0; i < 8; ++i) lo[i] = (E)g[i], hi[i] = (E)g[i + 8];
            E *to = (E *)out.p + row * out.row + head * out.head;
            if (p.a >= 0) store8(to + 8 * p.a, lo);
            if (p.b >= 0) store8(to + 8 * p.b, hi);
        }
    }
    if (!a.grad_q_weight && !a.grad_k_weight) return;
    // sums over the workgroup's heads, queries and keys apart, in their order
    const int slot = threadIdx.x / LANES, slots = blockDim.x / LANES;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (p.a >= 0) sums[slot * WIDE + 8 * p.a + i] = gw[i];
        if (p.b >= 0) sums[slot * WIDE + 8 * p.b + i] = gw[i + 8];
    }
    __syncthreads();
    float *to = a.partial + (int64_t)(blockIdx.y * gridDim.x + blockIdx.x) * 2 * a.dim;
    const int first = blockIdx.y * share.heads, used = share.heads * share.rows < slots ? share.heads * share.rows : slots;
    for (int i = threadIdx.x; i < 2 * a.dim; i += blockDim.x) {
        const int d = i % a.dim, begin = i < a.dim ? 0 : a.q_heads, end = i < a.dim ? a.q_heads : units;
        float s = 0.0f;
        for (int u = 0; u < used; ++u) {
            const int unit = first + u % share.heads;
            if (unit >= begin && unit < end) s += sums[u * WIDE + d];
        }
        to[i] = s;
    }
}

// 16 columns a workgroup, each in 64 parts.
__global__ __launch_bounds__(1024) void head_rope_gw_kernel(const float *partial, float *q_weight, float *k_weight, int parts, int dim)
{
    __shared__ double sums[64][17];
    const int column = blockIdx.x * 16 + threadIdx.x % 16, part = threadIdx.x / 16;
    double s = 0.0;
    if (column < 2 * dim)
#pragma unroll 8
        for (int i = part; i < parts; i += 64) s += (double)partial[(int64_t)i * 2 * dim + column];
    sums[part][threadIdx.x % 16] = s;
    __syncthreads();
    if (part != 0 || column >= 2 * dim) return;
    for (int i = 1; i < 64; ++i) s += sums[i][threadIdx.x % 16];
    float *to = column < dim ? q_weight : k_weight;
    if (to) to[column % dim] = (float)s;
}

int lanes_of(int dim) { return dim <= 16 ? 1 : dim <= 32 ? 2 : dim <= 64 ? 4 : dim <= 128 ? 8 : 16; }
// Several rows of few heads, or part of a row of more than 256 threads' worth; whole waves.
Share share_of(int rows, int units, int dim)
{
    const int lanes = lanes_of(dim), row = units * lanes;
    Share s;
    s.blocks = (row + kThreads - 1) / kThreads;
    s.heads = (units + s.blocks - 1) / s.blocks;
    s.rows = s.blocks > 1 ? 1 : 256 / row < 1 ? 1 : 256 / row < kRows ? 256 / row : kRows;
    if (s.rows > rows) s.rows = rows;
    s.threads = (s.rows * s.heads * lanes + 63) / 64 * 64;
    return s;
}
// Workgroups of the backward pass along the rows: three a compute unit, as many as its registers hold (four take a third longer).
int row_groups(int rows, const Share &s)
{
    const int groups = (rows + s.rows - 1) / s.rows, most = 768 / s.blocks > 1 ? 768 / s.blocks : 1;
    return groups < most ? groups : most;
}

template <class E, int LANES>
hipError_t forward(const DsqRopeArgs &a, hipStream_t stream)
{
    const Share s = share_of(a.rows, a.q_heads + a.kv_heads + (a.cache.k ? a.kv_heads : 0), a.dim);
    head_rope_kernel<E, LANES><<<dim3((a.rows + s.rows - 1) / s.rows, s.blocks), s.threads, 0, stream>>>(a, s);
    return hipGetLastError();
}
template <class E, int LANES>
hipError_t backward(const DsqRopeBwdArgs &a, hipStream_t stream)
{
    const Share s = share_of(a.rows, a.q_heads + a.kv_heads, a.dim);
    const int groups = row_groups(a.rows, s);
    head_rope_bwd_kernel<E, LANES><<<dim3(groups, s.blocks), s.threads, 0, stream>>>(a, s);
    if (const hipError_t e = hipGetLastError()) return e;
    if (a.grad_q_weight || a.grad_k_weight)
        head_rope_gw_kernel<<<(2 * a.dim + 15) / 16, 1024, 0, stream>>>(a.partial, a.grad_q_weight, a.grad_k_weight, groups * s.blocks, a.dim);
    return hipGetLastError();
}

template <class E>
hipError_t of_dim(const DsqRopeArgs &a, hipStream_t stream)
{
    switch (lanes_of(a.dim)) {
    case 1: return forward<E, 1>(a, stream);
    case 2: return forward<E, 2>(a, stream);
    case 4: return forward<E, 4>(a, stream);
    case 8: return forward<E, 8>(a, stream);
    default: return forward<E, 16>(a, stream);
    }
}
template <class E>
hipError_t of_dim(const DsqRopeBwdArgs &a, hipStream_t stream)
{
    switch (lanes_of(a.dim)) {
    case 1: return backward<E, 1>(a, stream);
    case 2: return backward<E, 2>(a, stream);
    case 4: return backward<E, 4>(a, stream);
    case 8: return backward<E, 8>(a, stream);
    default: return backward<E, 16>(a, stream);
    }
}

template <class A>
hipError_t of_type(const A &a, int type, hipStream_t stream)
{
    if (type == DSQ_T_F32) return of_dim<float>(a, stream);
    if (type == DSQ_T_F16) return of_dim<_Float16>(a, stream);
    return of_dim<__bf16>(a, stream);
}

}  // namespace

int dsq_rope_bwd_parts(int rows, int q_heads, int kv_heads, int dim)
{
    const Share s = share_of(rows, q_heads + kv_heads, dim);
    return row_groups(rows, s) * s.blocks;
}
hipError_t dsq_launch_qk_norm_rope(const DsqRopeArgs &a, int type, hipStream_t stream) { return of_type(a, type, stream); }
hipError_t dsq_launch_qk_norm_rope_bwd(const DsqRopeBwdArgs &a, int type, hipStream_t stream) { return of_type(a, type, stream); }
