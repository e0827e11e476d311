// RMS norm of rows with the residual's addition, its rows as floats and as 8-bit codes, and its backward pass.
//
//   h = x + residual (binary32, rounded to the type), r = 1 / sqrt(mean h^2 + eps), y = h * r * w
//   codes: amax = max |h * w|, code = rint(127 * h * w / amax), scale = r * amax / 127
//
// r cancels in a code, so sum of squares and amax come out of one pass over registers and a code is decided by h and
// w alone.  Squares, products and the quotient are formed in binary64, in which the product of two binary32 numbers is
// exact: nothing over- or underflows over the whole range of the types, y is rounded once, and a code is the
// correctly rounded quotient.
//
//   backward, t = gy * w, n = h * r:  gx = r * (t - n * mean(t * n)) + gsum,  gw = sum over rows of gy * n
//
// Both read and write every tensor once; bound by HBM bandwidth, and by latency for a few rows.
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

// The code of the product p: its quotient by the step amax / 127, rounded to the nearest integer.  p * inv is within
// 2^-44 of the quotient; only one that near to a half is divided out.
__device__ __forceinline__ int code_of(double p, double inv, double amax)
{
    double t = p * inv;
    const double n = rint(t);
    if (__builtin_expect(fabs(t - n) > 0.5 - 0x1p-40, 0)) return (int)rint(127.0 * p / amax);
    return (int)n;
}

// Elements a thread keeps: VPT vectors of V.  Thread `t` of the TPR of a row has vectors t, t + TPR, ...
template <int T, int TPR, int VPT>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rms_norm_kernel(DsqNormArgs a)
{
    typedef typename Element<T>::type E;
    constexpr int V = 16 / (int)sizeof(E);
    constexpr int THREADS = TPR < 256 ? 256 : TPR, RPB = THREADS / TPR, WAVES = THREADS / 64;
    __shared__ double part[2][WAVES];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    const bool live = row < a.rows;
    const E *x = (const E *)a.x + row * a.x_stride;
    const E *res = a.residual ? (const E *)a.residual + row * a.residual_stride : nullptr;
    const E *wt = (const E *)a.weight;

    float h[VPT * V], w[VPT * V];
    double ss = 0.0, amax = 0.0;
    float mark = 0.0f;       // NaN once a weight is not finite
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int at = (t + j * TPR) * V;
        Side<E, V> xv = {}, rv = {}, wv;
#pragma unroll
        for (int v = 0; v < V; ++v) wv.at[v] = (E)1.0f;
        if (live) {
            if (at + V <= a.dim) {
                xv = load_side<E, V>(x + at);
                if (res) rv = load_side<E, V>(res + at);
                if (wt) wv = load_side<E, V>(wt + at);
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (at + v < a.dim) {
                        xv.at[v] = x[at + v];
                        if (res) rv.at[v] = res[at + v];
                        if (wt) wv.at[v] = wt[at + v];
                    }
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const E s = res ? (E)((float)xv.at[v] + (float)rv.at[v]) : xv.at[v];
            h[j * V + v] = (float)s;
            w[j * V + v] = (float)wv.at[v];
            mark = __builtin_fmaf(w[j * V + v], 0.0f, mark);
            xv.at[v] = s;
            ss += (double)h[j * V + v] * (double)h[j * V + v];
            amax = fmax(amax, fabs((double)h[j * V + v] * (double)w[j * V + v]));
        }
        if (a.sum && live) {
            E *to = (E *)a.sum + row * a.dim + at;
            if (at + V <= a.dim) store_side<E, V>(to, xv);
            else
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (at + v < a.dim) to[v] = xv.at[v];
        }
    }
    ss = lane_sum(ss, TPR < 64 ? TPR : 64);
    mark = lane_sum(mark, TPR < 64 ? TPR : 64);
    if (a.codes) amax = lane_max(amax, TPR < 64 ? TPR : 64);
    if (TPR > 64) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) { part[0][wave] = ss; part[1][wave] = mark == 0.0f ? amax : __builtin_inf(); }
        __syncthreads();
        ss = 0.0; amax = 0.0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) { ss += part[0][i]; amax = fmax(amax, part[1][i]); }
    } else if (mark != 0.0f) {
        amax = __builtin_inf();
    }
    if (!live) return;
    const double r = 1.0 / sqrt(ss / (double)a.dim + (double)a.eps);
    // (fmax passes over a NaN: a row that holds one, or an infinity, is marked by its sum of squares, a weight by an amax of
    // infinity)
    const bool bad = !(ss <= 1.7e308 && amax <= 1.7e308);
    const double inv = amax > 0.0 && !bad ? 127.0 / amax : 0.0;
    if (t == 0) {
        if (a.rstd) a.rstd[row] = (float)r;
        if (a.codes) a.scales[row] = bad ? __builtin_nanf("") : (float)(amax * r / 127.0);
    }
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const int at = (t + j * TPR) * V;
        if (a.y && at < a.dim) {
            Side<E, V> yv;
#pragma unroll
            for (int v = 0; v < V; ++v) yv.at[v] = (E)(float)((double)h[j * V + v] * (double)w[j * V + v] * r);
            E *to = (E *)a.y + row * a.dim + at;
            if (at + V <= a.dim) store_side<E, V>(to, yv);
            else
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (at + v < a.dim) to[v] = yv.at[v];
        }
        if (a.codes && at < a.code_pitch) {
            Side<int8_t, V> cv;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                // (h is 0 past the row's end)
                cv.at[v] = inv == 0.0 ? 0 : (int8_t)code_of((double)h[j * V + v] * (double)w[j * V + v], inv, amax);
            }
            store_side<int8_t, V>(a.codes + row * a.code_pitch + at, cv);
        }
    }
    // what lies between the row's end and its pitch, past what the threads hold
    if (a.codes)
        for (int64_t at = (int64_t)TPR * VPT * V + t; at < a.code_pitch; at += TPR) a.codes[row * a.code_pitch + at] = 0;
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
template <int T, int TPR, int VPT>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rms_norm_bwd_kernel(DsqNormBwdArgs a)
{
    typedef typename Element<T>::type E;
    constexpr int V = 16 / (int)sizeof(E);
    constexpr int THREADS = TPR < 256 ? 256 : TPR, RPB = THREADS / TPR, WAVES = THREADS / 64;
    __shared__ float part[2][WAVES];
    __shared__ float rows_gw[RPB > 1 ? TPR * VPT * V : 1];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    float w[VPT * V], gw[VPT * V];
#pragma unroll
    for (int i = 0; i < VPT * V; ++i) {
        const int at = (t + (i / V) * TPR) * V + i % V;
        w[i] = a.weight && at < a.dim ? (float)((const E *)a.weight)[at] : 1.0f;
        gw[i] = 0.0f;
    }
    int flip = 0;
    for (int64_t base = (int64_t)blockIdx.x * RPB; base < a.rows; base += (int64_t)gridDim.x * RPB) {
        const int64_t row = base + sub;
        const bool live = row < a.rows;
        const E *h = (const E *)a.h + row * a.h_stride, *gy = (const E *)a.grad_y + row * a.grad_y_stride;
        const E *gs = a.grad_sum ? (const E *)a.grad_sum + row * a.grad_sum_stride : nullptr;
        const float r = live ? a.rstd[row] : 0.0f;
        Side<E, V> hv[VPT], gv[VPT], sv[VPT];
        float along = 0.0f;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int at = (t + j * TPR) * V;
            hv[j] = {}; gv[j] = {}; sv[j] = {};
            if (live) {
                if (at + V <= a.dim) {
                    hv[j] = load_side<E, V>(h + at);
                    gv[j] = load_side<E, V>(gy + at);
                    if (gs) sv[j] = load_side<E, V>(gs + at);
                } else {
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        if (at + v < a.dim) {
                            hv[j].at[v] = h[at + v];
                            gv[j].at[v] = gy[at + v];
                            if (gs) sv[j].at[v] = gs[at + v];
                        }
                }
            }
        }
#pragma unroll
        for (int j = 0; j < VPT; ++j)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float n = (float)hv[j].at[v] * r, g = (float)gv[j].at[v];
                gw[j * V + v] = __builtin_fmaf(g, n, gw[j * V + v]);
                along = __builtin_fmaf(g * w[j * V + v], n, along);
            }
        along = lane_sum(along, TPR < 64 ? TPR : 64);
        if (TPR > 64) {
            // (two areas in turn: one barrier a row)
            if ((threadIdx.x & 63) == 0) part[flip][threadIdx.x >> 6] = along;
            __syncthreads();
            along = 0.0f;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) along += part[flip][i];
            flip ^= 1;
        }
        along /= (float)a.dim;
        if (!live) continue;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const int at = (t + j * TPR) * V;
            Side<E, V> ov;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float n = (float)hv[j].at[v] * r, g = (float)gv[j].at[v];
                ov.at[v] = (E)__builtin_fmaf(r, __builtin_fmaf(-n, along, g * w[j * V + v]), (float)sv[j].at[v]);
            }
            E *to = (E *)a.grad_x + row * a.dim + at;
            if (at + V <= a.dim) store_side<E, V>(to, ov);
            else
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (at + v < a.dim) to[v] = ov.at[v];
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
        for (int at = threadIdx.x; at < a.dim; at += THREADS) a.partial[(size_t)blockIdx.x * a.dim + at] = rows_gw[at];
    } else {
#pragma unroll
        for (int i = 0; i < VPT * V; ++i) {
            const int at = (t + (i / V) * TPR) * V + i % V;
            if (at < a.dim) a.partial[(size_t)blockIdx.x * a.dim + at] = gw[i];
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
    float *gw = a.partial + (size_t)blockIdx.x * a.dim;
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

// grad_weight[c] = sum over the workgroups' partial rows: 64 columns a workgroup, 16 strips of rows joined in LDS.
__global__ __launch_bounds__(1024) void rms_norm_gw_kernel(const float *partial, float *gw, int parts, int dim)
{
    __shared__ double strip[16][64];
    const int lane = threadIdx.x & 63, s = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    double sum = 0.0;
    if (c < dim)
        for (int p = s; p < parts; p += 16) sum += (double)partial[(size_t)p * dim + c];
    strip[s][lane] = sum;
    __syncthreads();
    if (s == 0 && c < dim) {
        for (int i = 1; i < 16; ++i) sum += strip[i][lane];
        gw[c] = (float)sum;
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
    for (int tpr : {16, 64, 256, 1024})
        for (int vpt : {1, 2, 4})
            if (vectors <= tpr * vpt) return {tpr, vpt};
    return {0, 0};
}

template <int T, int TPR, int VPT>
hipError_t launch_fwd(const DsqNormArgs &a, hipStream_t stream)
{
    constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
    rms_norm_kernel<T, TPR, VPT><<<(unsigned)((a.rows + (int64_t)RPB - 1) / RPB), TPR < 256 ? 256 : TPR, 0, stream>>>(a);
    return hipGetLastError();
}
template <int T, int TPR, int VPT>
hipError_t launch_bwd(const DsqNormBwdArgs &a, int parts, hipStream_t stream)
{
    rms_norm_bwd_kernel<T, TPR, VPT><<<parts, TPR < 256 ? 256 : TPR, 0, stream>>>(a);
    return hipGetLastError();
}

// f(threads of a row, vectors of a thread) with both as constants.
template <class F>
hipError_t with_shape(Shape s, F f)
{
#define DSQ_SHAPE(TPR, VPT) \
    if (s.tpr == TPR && s.vpt == VPT) return f(std::integral_constant<int, TPR>(), std::integral_constant<int, VPT>());
    DSQ_SHAPE(16, 1) DSQ_SHAPE(16, 2) DSQ_SHAPE(16, 4) DSQ_SHAPE(64, 2) DSQ_SHAPE(64, 4) DSQ_SHAPE(256, 2) DSQ_SHAPE(256, 4)
    DSQ_SHAPE(1024, 2) DSQ_SHAPE(1024, 4)
#undef DSQ_SHAPE
    return hipErrorInvalidValue;
}

template <int T>
hipError_t launch_fwd_of(const DsqNormArgs &a, hipStream_t stream)
{
    const Shape s = shape_of(a.dim, T);
    if (s.tpr == 0) {
        rms_norm_long_kernel<T><<<a.rows, 1024, 0, stream>>>(a);
        return hipGetLastError();
    }
    return with_shape(s, [&](auto tpr, auto vpt) { return launch_fwd<T, tpr.value, vpt.value>(a, stream); });
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
        e = with_shape(s, [&](auto tpr, auto vpt) { return launch_bwd<T, tpr.value, vpt.value>(a, parts, stream); });
    }
    if (e != hipSuccess || !a.grad_weight) return e;
    rms_norm_gw_kernel<<<(a.dim + 63) / 64, 1024, 0, stream>>>(a.partial, a.grad_weight, parts, a.dim);
    return hipGetLastError();
}

}  // namespace

int dsq_rms_norm_bwd_parts(int rows, int dim, int type)
{
    const Shape s = shape_of(dim, type);
    const int rpb = s.tpr == 0 || s.tpr >= 256 ? 1 : 256 / s.tpr;
    const int64_t groups = ((int64_t)rows + rpb - 1) / rpb;
    return (int)(groups < 512 ? groups : 512);
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
