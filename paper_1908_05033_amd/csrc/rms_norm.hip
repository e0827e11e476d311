// RMS norm of rows with the residual's addition, its rows as floats and as 8-bit codes, and its backward pass.
//
//   h = x + residual (binary32, rounded to the type), r = 1 / sqrt(mean h^2 + eps), y = h * r * w
//   codes: amax = max |h * w|, code = rint(127 * h * w / amax), scale = r * amax / 127
//
// r cancels in a code, so sum of squares and amax come out of one pass over registers and a code is decided by h and
// w alone.  Squares, products and the quotient are formed in binary64, in which the product of two binary32 numbers is
// exact: nothing over- or underflows over the whole range of the types, y is rounded once, and a code is the
// correctly rounded quotient (one beside a half is decided exactly, code_of).
//
//   backward, t = gy * w, n = h * r:  gx = r * (t - n * mean(t * n)) + gsum,  gw = sum over rows of gy * n
//
// Both read and write every tensor once; bound by HBM bandwidth, and by latency for a few rows: 8192 rows of 4096 bfloat16 take 48 us
// forward (5.6 TB/s) and 53 + 5 us backward (5.1 TB/s), 2048 rows to codes 17 us (3.4 TB/s), one row 3.6 us.
#include <type_traits>

#include "lm_device.h"

namespace {

__device__ __forceinline__ double lane_sum(double v, int lanes)
{
    for (int off = lanes / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}
__device__ __forceinline__ float lane_sum(float v, int lanes)
{
    for (int off = lanes / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}
__device__ __forceinline__ double lane_max(double v, int lanes)
{
    for (int off = lanes / 2; off > 0; off >>= 1) v = fmax(v, __shfl_xor(v, off));
    return v;
}

// The code of the product p: its quotient by the step amax / 127, rounded to the nearest integer, halves to even.  p * inv is within
// 2^-44 of the quotient; one that near to a half, whole + 1/2, is decided by the sign of 254 |p| - (2 whole + 1) amax.  p and amax
// have 48 significant bits, so a factor of 8 bits leaves each product a few bits longer than a binary64 number: both are taken with
// what their rounding left, and their difference is exact.
__device__ __forceinline__ int code_of(double p, double inv, double amax)
{
    const double t = p * inv;
    const double n = rint(t);
    if (__builtin_expect(fabs(t - n) > 0.5 - 0x1p-40, 0)) {
        const double whole = floor(fabs(t)), odd = 2.0 * whole + 1.0, size = fabs(p);
        const double a = 254.0 * size, b = odd * amax;
        const double past = (a - b) + (__builtin_fma(254.0, size, -a) - __builtin_fma(odd, amax, -b));
        const int code = (int)whole, up = past > 0.0 || (past == 0.0 && (code & 1));
        return p < 0.0 ? -(code + up) : code + up;
    }
    return (int)n;
}

// 16 bytes of a row, V elements as they lie in memory (kept so while they are under way: taken apart they would fill a register each).
template <class E>
struct Raw {
    uint64_t lo, hi;
    __device__ __forceinline__ float operator[](int v) const
    {
        constexpr int PER = 8 / (int)sizeof(E);
        const uint64_t half = v < PER ? lo : hi;
        const uint32_t word = (uint32_t)(half >> (v % PER * 8 * (int)sizeof(E) / 32 * 32));
        if constexpr (sizeof(E) == 4) return __uint_as_float(word);
        else if constexpr (__is_same(E, __bf16)) return __uint_as_float(v % 2 ? word & 0xFFFF0000u : word << 16);
        else {
            const uint16_t bits = (uint16_t)(v % 2 ? word >> 16 : word);
            return (float)__builtin_bit_cast(_Float16, bits);
        }
    }
};

// Elements at .. at + V - 1 of a row of `dim` elements, 0 past its end, in two parts.  The load stands behind no branch and is not
// touched (it would be waited for): past the end it takes the row's last V.  in_row() moves them down, where they are used.
// WHOLE: dim is a multiple of V, and a vector lies in the row or behind it.
template <class E, int V, bool WHOLE>
__device__ __forceinline__ Raw<E> load_raw(const E *row, int at, int dim)
{
    Raw<E> r = {0, 0};
    if (WHOLE || dim >= V) {
        const Side<uint64_t, 2> s = load_side<uint64_t, 2>((const uint64_t *)(row + (at < dim - V ? at : dim - V)));
        r.lo = s.at[0];
        r.hi = s.at[1];
    } else {
        Side<E, V> e;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const E x = row[at + v < dim ? at + v : 0];
            e.at[v] = at + v < dim ? x : (E)0.0f;
        }
        __builtin_memcpy(&r, &e, 16);
    }
    return r;
}
template <class E, int V, bool WHOLE>
__device__ __forceinline__ Raw<E> in_row(Raw<E> r, int at, int dim)
{
    const int back = at + V - dim;                  // elements before `at` among the row's last V
    if (WHOLE) {
        if (back > 0) r.lo = r.hi = 0;
    } else if (dim >= V) {
        const int n = 8 * (int)sizeof(E) * (back < 0 ? 0 : back < V ? back : V);
        // (without branches: 0, 64 and 128 are moves of whole halves)
        const uint64_t lo = n >= 128 ? 0 : n >= 64 ? r.hi : r.lo, hi = n >= 64 ? 0 : r.hi;
        r.lo = lo >> (n & 63) | hi << 1 << (63 - (n & 63));
        r.hi = hi >> (n & 63);
    }
    return r;
}
template <class E, int V, bool WHOLE>
__device__ __forceinline__ void store_in_row(E *row, int at, int dim, const Side<E, V> &v)
{
    if (at >= dim) return;
    if (WHOLE || at + V <= dim) store_side<E, V>(row + at, v);
    else
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (at + i < dim) row[at + i] = v.at[i];
}

// Elements a thread keeps: VPT vectors of V.  Thread `t` of the TPR of a row has vectors t, t + TPR, ...; a workgroup takes
// row groups b, b + gridDim.x, ..., with the next group's rows under way while one is worked on.
template <int T, int TPR, int VPT, bool WHOLE>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR, 4) void rms_norm_kernel(DsqNormArgs a)
{
    typedef typename Element<T>::type E;
    constexpr int V = 16 / (int)sizeof(E), N = VPT * V;
    constexpr int THREADS = TPR < 256 ? 256 : TPR, RPB = THREADS / TPR, WAVES = THREADS / 64;
    __shared__ double part[2][2][WAVES];      // (rows of more than a wave)
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    if (VPT > 1) __builtin_assume(a.dim > TPR * V);
    float w[N];
    float mark = 0.0f;       // NaN once a weight is not finite
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        Raw<E> wv = {0, 0};
        if (a.weight) wv = in_row<E, V, WHOLE>(load_raw<E, V, WHOLE>((const E *)a.weight, (t + j * TPR) * V, a.dim), (t + j * TPR) * V, a.dim);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            w[j * V + v] = a.weight ? wv[v] : 1.0f;
            mark = __builtin_fmaf(w[j * V + v], 0.0f, mark);
        }
    }
    Raw<E> xv[VPT], rv[VPT] = {};
    auto load = [&](int64_t row) __attribute__((always_inline)) {
        if (row >= a.rows) row = a.rows - 1;                    // (not stored)
        const E *x = (const E *)a.x + row * a.x_stride;
#pragma unroll
        for (int j = 0; j < VPT; ++j) xv[j] = load_raw<E, V, WHOLE>(x, (t + j * TPR) * V, a.dim);
        if (a.residual) {
            const E *res = (const E *)a.residual + row * a.residual_stride;
#pragma unroll
            for (int j = 0; j < VPT; ++j) rv[j] = load_raw<E, V, WHOLE>(res, (t + j * TPR) * V, a.dim);
        }
    };
    int flip = 0;
    constexpr bool AHEAD = VPT == 1;                            // (more vectors leave no registers for the next row's)
    if (AHEAD) load((int64_t)blockIdx.x * RPB + sub);
    for (int64_t base = (int64_t)blockIdx.x * RPB; base < a.rows; base += (int64_t)gridDim.x * RPB) {
        const int64_t row = base + sub;
        const bool live = row < a.rows;
        if (!AHEAD) load(row);
        int dim = a.dim;
        asm volatile("" : "+s"(dim));                           // (which elements exist is found again for each row: kept, the answers spill)
        if (VPT > 1) __builtin_assume(dim > TPR * V);
        float h[N];
        double ss = 0.0, amax = 0.0;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int at = (t + j * TPR) * V;
            const Raw<E> x = in_row<E, V, WHOLE>(xv[j], at, dim), res = in_row<E, V, WHOLE>(rv[j], at, dim);
            Side<E, V> sv;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const E s = (E)(a.residual ? x[v] + res[v] : x[v]);
                const float f = (float)s;
                sv.at[v] = s;
                h[j * V + v] = f;
                ss = __builtin_fma((double)f, (double)f, ss);
                amax = fmax(amax, fabs((double)f * (double)w[j * V + v]));
            }
            if (a.sum && live) store_in_row<E, V, WHOLE>((E *)a.sum + row * a.dim, at, dim, sv);
        }
        if (AHEAD) load(row + (int64_t)gridDim.x * RPB);
        if (mark != 0.0f) amax = __builtin_inf();
        ss = lane_sum(ss, TPR < 64 ? TPR : 64);
        if (a.codes) amax = lane_max(amax, TPR < 64 ? TPR : 64);
        if (TPR > 64) {
            // (two areas in turn: one barrier a row)
            const int wave = threadIdx.x >> 6;
            if ((threadIdx.x & 63) == 0) { part[flip][0][wave] = ss; part[flip][1][wave] = amax; }
            __syncthreads();
            ss = 0.0; amax = 0.0;
#pragma unroll
            for (int i = 0; i < TPR / 64; ++i) {
                ss += part[flip][0][sub * (TPR / 64) + i];
                amax = fmax(amax, part[flip][1][sub * (TPR / 64) + i]);
            }
            flip ^= 1;
        }
        const double r = 1.0 / sqrt(ss / (double)a.dim + (double)a.eps);
        // (fmax passes over a NaN: a row that holds one, or an infinity, is marked by its sum of squares, a weight by an amax of
        // infinity)
        const bool bad = !(ss <= 1.7e308 && amax <= 1.7e308);
        const double inv = amax > 0.0 && !bad ? 127.0 / amax : 0.0;
        if (t == 0 && live) {
            if (a.rstd) a.rstd[row] = (float)r;
            if (a.codes) a.scales[row] = bad ? __builtin_nanf("") : (float)(amax * r / 127.0);
        }
        if (!live) continue;
        if (a.y)
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const int at = (t + j * TPR) * V;
                Side<E, V> yv;
#pragma unroll
                for (int v = 0; v < V; ++v) yv.at[v] = (E)(float)((double)h[j * V + v] * (double)w[j * V + v] * r);
                store_in_row<E, V, WHOLE>((E *)a.y + row * a.dim, at, dim, yv);
            }
        if (a.codes) {
            const float inv32 = (float)inv;
#pragma unroll
            for (int j = 0; j < VPT; ++j) {
                const int at = (t + j * TPR) * V;
                Side<int8_t, V> cv;
                float near = 0.0f;
                // In binary32 the quotient is within 127 * 4 * 2^-24 < 2^-14 (product, 127 / amax, and theirs) unless amax is an extreme
                // number: nearer to a half, or with such a one, it is decided in binary64.  (h is 0 past the row's end.)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float q = h[j * V + v] * w[j * V + v] * inv32, n = rintf(q);
                    near = fmaxf(near, fabsf(q - n));
                    cv.at[v] = (int8_t)(int)n;
                }
                if (inv == 0.0 || inv > 0x1p100 || inv < 0x1p-100 || near > 0.5f - 0x1p-14f)
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        cv.at[v] = inv == 0.0 ? 0 : (int8_t)code_of((double)h[j * V + v] * (double)w[j * V + v], inv, amax);
                if (at < a.code_pitch) store_side<int8_t, V>(a.codes + row * a.code_pitch + at, cv);
            }
            // what lies between the row's end and its pitch, past what the threads hold
            for (int64_t at = (int64_t)TPR * VPT * V + t; at < a.code_pitch; at += TPR) a.codes[row * a.code_pitch + at] = 0;
        }
    }
}

// Rows longer than the registers of a workgroup: one workgroup a row, which reads the row a second time (from the
// sum where that is written) after the statistics.  Every element is read and written by one thread, so a `sum` in
// the place of an input does no harm.
template <int T>
__global__ __launch_bounds__(1024) void rms_norm_long_kernel(DsqNormArgs a)
{
    typedef typename Element<T>::type E;
    __shared__ double part[2][16];
    const int64_t row = blockIdx.x;
    const E *x = (const E *)a.x + row * a.x_stride;
    const E *res = a.residual ? (const E *)a.residual + row * a.residual_stride : nullptr;
    const E *wt = (const E *)a.weight;
    E *sum = a.sum ? (E *)a.sum + row * a.dim : nullptr;
    double ss = 0.0, amax = 0.0;
    float mark = 0.0f;
    for (int at = threadIdx.x; at < a.dim; at += 1024) {
        const E s = res ? (E)((float)x[at] + (float)res[at]) : x[at];
        if (sum) sum[at] = s;
        const double hd = (double)(float)s;
        ss += hd * hd;
        const float w = wt ? (float)wt[at] : 1.0f;
        mark = __builtin_fmaf(w, 0.0f, mark);
        amax = fmax(amax, fabs(hd * (double)w));
    }
    if (mark != 0.0f) amax = __builtin_inf();
    ss = lane_sum(ss, 64);
    amax = lane_max(amax, 64);
    if ((threadIdx.x & 63) == 0) { part[0][threadIdx.x >> 6] = ss; part[1][threadIdx.x >> 6] = amax; }
    __syncthreads();
    ss = 0.0; amax = 0.0;
    for (int i = 0; i < 16; ++i) { ss += part[0][i]; amax = fmax(amax, part[1][i]); }
    const double r = 1.0 / sqrt(ss / (double)a.dim + (double)a.eps);
    const bool bad = !(ss <= 1.7e308 && amax <= 1.7e308);
    const double inv = amax > 0.0 && !bad ? 127.0 / amax : 0.0;
    if (threadIdx.x == 0) {
        if (a.rstd) a.rstd[row] = (float)r;
        if (a.codes) a.scales[row] = bad ? __builtin_nanf("") : (float)(amax * r / 127.0);
    }
    if (!a.y && !a.codes) return;
    const int64_t end = a.codes ? a.code_pitch : a.dim;
    for (int64_t at = threadIdx.x; at < end; at += 1024) {
        double p = 0.0;
        if (at < a.dim) {
            const E s = sum ? sum[at] : res ? (E)((float)x[at] + (float)res[at]) : x[at];
            p = (double)(float)s * (wt ? (double)(float)wt[at] : 1.0);
            if (a.y) ((E *)a.y)[row * a.dim + at] = (E)(float)(p * r);
        }
        if (a.codes) a.codes[row * a.code_pitch + at] = inv == 0.0 ? 0 : (int8_t)code_of(p, inv, amax);
    }
}

// Backward: workgroup b takes row groups b, b + gridDim.x, ..., its threads the same columns of each, and leaves the
// weight gradient of its rows in partial[b]; the rows' order within a workgroup and the workgroups' in the second kernel
// are fixed, so the result is the same every time.
template <int T, int TPR, int VPT, bool WHOLE>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR, 4) void rms_norm_bwd_kernel(DsqNormBwdArgs a)
{
    typedef typename Element<T>::type E;
    constexpr int V = 16 / (int)sizeof(E);
    constexpr int THREADS = TPR < 256 ? 256 : TPR, RPB = THREADS / TPR, WAVES = THREADS / 64;
    __shared__ float part[2][WAVES];
    __shared__ float rows_gw[RPB > 1 ? TPR * VPT * V : 1];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    if (VPT > 1) __builtin_assume(a.dim > TPR * V);
    float *partial = gridDim.x == 1 ? a.grad_weight : a.partial + (size_t)blockIdx.x * a.dim;
    float w[VPT * V], gw[VPT * V];
#pragma unroll
    for (int i = 0; i < VPT * V; ++i) {
        const int at = (t + (i / V) * TPR) * V + i % V;
        w[i] = a.weight && at < a.dim ? (float)((const E *)a.weight)[at] : 1.0f;
        gw[i] = 0.0f;
    }
    Raw<E> hv[VPT], gv[VPT], sv[VPT] = {};
    float rs;
    auto load = [&](int64_t row) __attribute__((always_inline)) {
        if (row >= a.rows) row = a.rows - 1;                    // (met by an r of 0 and not stored)
        rs = a.rstd[row];
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int at = (t + j * TPR) * V;
            hv[j] = load_raw<E, V, WHOLE>((const E *)a.h + row * a.h_stride, at, a.dim);
            gv[j] = load_raw<E, V, WHOLE>((const E *)a.grad_y + row * a.grad_y_stride, at, a.dim);
            if (a.grad_sum) sv[j] = load_raw<E, V, WHOLE>((const E *)a.grad_sum + row * a.grad_sum_stride, at, a.dim);
        }
    };
    int flip = 0;
    constexpr bool AHEAD = VPT == 1;                            // (more vectors leave no registers for the next row's)
    if (AHEAD) load((int64_t)blockIdx.x * RPB + sub);
    for (int64_t base = (int64_t)blockIdx.x * RPB; base < a.rows; base += (int64_t)gridDim.x * RPB) {
        const int64_t row = base + sub;
        const bool live = row < a.rows;
        if (!AHEAD) load(row);
        int dim = a.dim;
        asm volatile("" : "+s"(dim));                           // (as in the forward pass)
        if (VPT > 1) __builtin_assume(dim > TPR * V);
        const float r = live ? rs : 0.0f;
        float n[VPT * V], gw_of[VPT * V];
        float along = 0.0f;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int at = (t + j * TPR) * V;
            const Raw<E> hr = in_row<E, V, WHOLE>(hv[j], at, dim), gr = in_row<E, V, WHOLE>(gv[j], at, dim);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int i = j * V + v;
                const float g = live ? gr[v] : 0.0f;
                n[i] = live ? hr[v] * r : 0.0f;
                gw[i] = __builtin_fmaf(g, n[i], gw[i]);
                gw_of[i] = g * w[i];
                along = __builtin_fmaf(gw_of[i], n[i], along);
            }
        }
        Raw<E> sw[VPT];
#pragma unroll
        for (int j = 0; j < VPT; ++j) sw[j] = sv[j];
        if (AHEAD) load(row + (int64_t)gridDim.x * RPB);
        along = lane_sum(along, TPR < 64 ? TPR : 64);
        if (TPR > 64) {
            // (two areas in turn: one barrier a row)
            if ((threadIdx.x & 63) == 0) part[flip][threadIdx.x >> 6] = along;
            __syncthreads();
            along = 0.0f;
#pragma unroll
            for (int i = 0; i < TPR / 64; ++i) along += part[flip][sub * (TPR / 64) + i];
            flip ^= 1;
        }
        along /= (float)a.dim;
        if (!live) continue;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int at = (t + j * TPR) * V;
            const Raw<E> s = in_row<E, V, WHOLE>(sw[j], at, dim);
            Side<E, V> ov;
#pragma unroll
            for (int v = 0; v < V; ++v)
                ov.at[v] = (E)__builtin_fmaf(r, __builtin_fmaf(-n[j * V + v], along, gw_of[j * V + v]), s[v]);
            store_in_row<E, V, WHOLE>((E *)a.grad_x + row * a.dim, at, dim, ov);
        }
    }
    if (!a.grad_weight) return;
    if (RPB > 1) {
        // the row slots of the workgroup add up one after the other
        for (int s = 0; s < RPB; ++s) {
            if (sub == s)
#pragma unroll
                for (int i = 0; i < VPT * V; ++i) {
                    const int at = (t + (i / V) * TPR) * V + i % V;
                    rows_gw[at] = s == 0 ? gw[i] : rows_gw[at] + gw[i];
                }
            __syncthreads();
        }
        for (int at = threadIdx.x; at < a.dim; at += THREADS) partial[at] = rows_gw[at];
    } else {
#pragma unroll
        for (int i = 0; i < VPT * V; ++i) {
            const int at = (t + (i / V) * TPR) * V + i % V;
            if (at < a.dim) partial[at] = gw[i];
        }
    }
}

// Rows longer than the registers of a workgroup: each is read twice, and the weight gradient of the workgroup's rows
// is kept in its row of partial sums, every column by one thread.
template <int T>
__global__ __launch_bounds__(1024) void rms_norm_bwd_long_kernel(DsqNormBwdArgs a)
{
    typedef typename Element<T>::type E;
    __shared__ float part[16];
    const E *w = (const E *)a.weight;
    float *gw = gridDim.x == 1 ? a.grad_weight : a.partial + (size_t)blockIdx.x * a.dim;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const E *h = (const E *)a.h + row * a.h_stride, *gy = (const E *)a.grad_y + row * a.grad_y_stride;
        const E *gs = a.grad_sum ? (const E *)a.grad_sum + row * a.grad_sum_stride : nullptr;
        const float r = a.rstd[row];
        float along = 0.0f;
        for (int at = threadIdx.x; at < a.dim; at += 1024) {
            const float n = (float)h[at] * r, g = (float)gy[at];
            if (a.grad_weight) gw[at] = row == blockIdx.x ? g * n : __builtin_fmaf(g, n, gw[at]);
            along = __builtin_fmaf(g * (w ? (float)w[at] : 1.0f), n, along);
        }
        along = lane_sum(along, 64);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = along;
        __syncthreads();
        along = 0.0f;
        for (int i = 0; i < 16; ++i) along += part[i];
        along /= (float)a.dim;
        for (int at = threadIdx.x; at < a.dim; at += 1024) {
            const float n = (float)h[at] * r, g = (float)gy[at];
            const float s = gs ? (float)gs[at] : 0.0f;
            ((E *)a.grad_x)[row * a.dim + at] = (E)__builtin_fmaf(r, __builtin_fmaf(-n, along, g * (w ? (float)w[at] : 1.0f)), s);
        }
    }
}

// grad_weight[c] = sum over the workgroups' partial rows: 16 columns a workgroup, 64 strips of rows, joined in the waves and then in
// LDS.  Latency bound: few columns a workgroup leave a thread few rows one after the other.
__global__ __launch_bounds__(1024) void rms_norm_gw_kernel(const float *partial, float *gw, int parts, int dim)
{
    __shared__ double strip[16][16];
    const int c = threadIdx.x & 15, s = threadIdx.x >> 4, column = blockIdx.x * 16 + c;
    double sum = 0.0;
    if (column < dim) {
#pragma unroll 8
        for (int p = s; p < parts; p += 64) sum += (double)partial[(size_t)p * dim + column];
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if ((threadIdx.x & 63) < 16) strip[threadIdx.x >> 6][c] = sum;
    __syncthreads();
    if (threadIdx.x < 16 && column < dim) {
        sum = 0.0;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += strip[i][c];
        gw[column] = (float)sum;
    }
}

// Threads of a row and the vectors each of them keeps.
struct Shape {
    int tpr, vpt;            // tpr = 0: the row is too long for a workgroup's registers
};
Shape shape_of(int dim, int type)
{
    const int V = type == DSQ_T_F32 ? 4 : 8;
    const int vectors = (dim + V - 1) / V;
    for (int tpr = 16; tpr <= 1024; tpr *= 2)
        if (vectors <= tpr) return {tpr, 1};
    for (int vpt = 2; vpt * V <= 16; vpt *= 2)
        if (vectors <= 1024 * vpt) return {1024, vpt};
    return {0, 0};
}

template <int T, int TPR, int VPT, bool WHOLE>
hipError_t launch_fwd(const DsqNormArgs &a, hipStream_t stream)
{
    constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
    // Up to 16 waves a compute unit, and more rows in turn with the next ones under way (us, 512 / 1024 / 2048 workgroups: 8192 rows of
    // 4096 bf16 52.0 / 51.6 / 53.6, 40000 of 128 11.6 / 11.0 / 11.7)
    const int64_t groups = (a.rows + (int64_t)RPB - 1) / RPB, most = TPR == 1024 ? 256 : 1024;
    rms_norm_kernel<T, TPR, VPT, WHOLE><<<(unsigned)(groups < most ? groups : most), TPR < 256 ? 256 : TPR, 0, stream>>>(a);
    return hipGetLastError();
}
template <int T, int TPR, int VPT, bool WHOLE>
hipError_t launch_bwd(const DsqNormBwdArgs &a, int parts, hipStream_t stream)
{
    rms_norm_bwd_kernel<T, TPR, VPT, WHOLE><<<parts, TPR < 256 ? 256 : TPR, 0, stream>>>(a);
    return hipGetLastError();
}

// f(threads of a row, vectors of a thread, whether a row ends with one) as constants: at most 16 elements a thread.
template <int T, class F>
hipError_t with_shape(Shape s, int dim, F f)
{
    hipError_t e = hipErrorInvalidValue;
    auto ends = [&](auto tpr, auto vpt) {
        e = dim % (T == DSQ_T_F32 ? 4 : 8) == 0 ? f(tpr, vpt, std::true_type()) : f(tpr, vpt, std::false_type());
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 1024> most;
    switch (s.tpr) {
    case 16: ends(std::integral_constant<int, 16>(), one); break;
    case 32: ends(std::integral_constant<int, 32>(), one); break;
    case 64: ends(std::integral_constant<int, 64>(), one); break;
    case 128: ends(std::integral_constant<int, 128>(), one); break;
    case 256: ends(std::integral_constant<int, 256>(), one); break;
    case 512: ends(std::integral_constant<int, 512>(), one); break;
    case 1024:
        if (s.vpt == 1) ends(most, one);
        if (s.vpt == 2) ends(most, std::integral_constant<int, 2>());
        if constexpr (T == DSQ_T_F32)
            if (s.vpt == 4) ends(most, std::integral_constant<int, 4>());
    }
    return e;
}

template <int T>
hipError_t launch_fwd_of(const DsqNormArgs &a, hipStream_t stream)
{
    const Shape s = shape_of(a.dim, T);
    if (s.tpr == 0) {
        rms_norm_long_kernel<T><<<a.rows, 1024, 0, stream>>>(a);
        return hipGetLastError();
    }
    return with_shape<T>(s, a.dim, [&](auto tpr, auto vpt, auto whole) { return launch_fwd<T, tpr.value, vpt.value, whole.value>(a, stream); });
}

template <int T>
hipError_t launch_bwd_of(const DsqNormBwdArgs &a, hipStream_t stream)
{
    const int parts = dsq_rms_norm_bwd_parts(a.rows, a.dim, T);
    const Shape s = shape_of(a.dim, T);
    hipError_t e;
    if (s.tpr == 0) {
        rms_norm_bwd_long_kernel<T><<<parts, 1024, 0, stream>>>(a);
        e = hipGetLastError();
    } else {
        e = with_shape<T>(s, a.dim, [&](auto tpr, auto vpt, auto whole) { return launch_bwd<T, tpr.value, vpt.value, whole.value>(a, parts, stream); });
    }
    if (e != hipSuccess || !a.grad_weight || parts == 1) return e;
    rms_norm_gw_kernel<<<(a.dim + 15) / 16, 1024, 0, stream>>>(a.partial, a.grad_weight, parts, a.dim);
    return hipGetLastError();
}

}  // namespace

int dsq_rms_norm_bwd_parts(int rows, int dim, int type)
{
    const Shape s = shape_of(dim, type);
    const int rpb = s.tpr == 0 || s.tpr >= 256 ? 1 : 256 / s.tpr;
    const int64_t groups = ((int64_t)rows + rpb - 1) / rpb;
    // More workgroups are more partial sums to write and to add (us, 384 / 512 / 768 / 1024: 8192 rows of 4096 bf16
    // 62.3 / 60.8 / 67.5 / 68.3; 512 / 768 / 1024: 20000 of 512 bf16 22.1 / 24.3 / 24.2); workgroups of 16 waves run one a compute unit
    const int64_t most = s.tpr == 0 || s.tpr == 1024 ? 256 : 512;
    return (int)(groups < most ? groups : most);
}

hipError_t dsq_launch_rms_norm(const DsqNormArgs &a, int type, hipStream_t stream)
{
    return type == DSQ_T_F32 ? launch_fwd_of<DSQ_T_F32>(a, stream)
           : type == DSQ_T_F16 ? launch_fwd_of<DSQ_T_F16>(a, stream) : launch_fwd_of<DSQ_T_BF16>(a, stream);
}

hipError_t dsq_launch_rms_norm_bwd(const DsqNormBwdArgs &a, int type, hipStream_t stream)
{
    return type == DSQ_T_F32 ? launch_bwd_of<DSQ_T_F32>(a, stream)
           : type == DSQ_T_F16 ? launch_bwd_of<DSQ_T_F16>(a, stream) : launch_bwd_of<DSQ_T_BF16>(a, stream);
}
