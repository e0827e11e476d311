// Rows times group-scaled 4-bit weights:  out[m][n] = sum over groups g of s[n][g] * sum over k in g of (code - z) x[m][k].
//
// The sum of a group runs on the 16x16x32 matrix instructions with exact operands: a code is converted to the type of
// x (a byte 0..15 is the e4m3 number code * 2^-9, which one instruction turns into bf16 or f16 times 2^9), binary32
// activations are cut into three bf16 terms, 8-bit rows meet the codes as bytes.  A matrix product with ones gives the
// group's sum of x for the zero points.  Groups are joined in binary32.
//
// A workgroup owns 16 output channels and 16 * MT rows; its waves share out the blocks of 128 input channels and join
// their sums in LDS, in a fixed order.
#include "lm_device.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef int v4i __attribute__((ext_vector_type(4)));

constexpr int ROWS_WAVES = 8;

// What a lane holds of a step of 32 channels of 16 rows: 8 consecutive channels of one row.
template <int XT>
struct Frag;
template <>
struct Frag<DSQ_T_BF16> {
    bf16x8 v;
};
template <>
struct Frag<DSQ_T_F16> {
    f16x8 v;
};
template <>
struct Frag<DSQ_T_F32> {
    float v[8];
};
template <>
struct Frag<DSQ_T_I8> {
    long v;
};

template <int XT>
__device__ __forceinline__ Frag<XT> load_frag(const void *row, int k, int K, bool live)
{
    Frag<XT> f = {};
    if constexpr (XT == DSQ_T_I8) {
        // (rows end with their pitch, a multiple of 128, and what lies behind K meets levels of 0)
        if (live) f.v = *reinterpret_cast<const long *>((const int8_t *)row + k);
    } else {
        typedef typename Element<XT>::type E;
        const E *p = (const E *)row + k;
        if (live && k + 8 <= K) {
            const Side<E, 8> s = load_side<E, 8>(p);
#pragma unroll
            for (int i = 0; i < 8; ++i) f.v[i] = s.at[i];
        } else if (live) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < K) f.v[i] = p[i];
        }
    }
    return f;
}

// The eight codes of a word as operand.
__device__ __forceinline__ bf16x8 codes_bf16(uint32_t w)
{
    const int lo = (int)(w & 0x0F0F0F0Fu), hi = (int)((w >> 4) & 0x0F0F0F0Fu);
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, true);
    return (bf16x8){a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
__device__ __forceinline__ f16x8 codes_f16(uint32_t w)
{
    const int lo = (int)(w & 0x0F0F0F0Fu), hi = (int)((w >> 4) & 0x0F0F0F0Fu);
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, true);
    const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, true);
    return (f16x8){a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
__device__ __forceinline__ long codes_i8(uint32_t w)
{
    const uint64_t lo = w & 0x0F0F0F0Fu, hi = (w >> 4) & 0x0F0F0F0Fu;
    return (long)(lo | hi << 32);
}

// x = t[0] + t[1] + t[2] exactly, eight significant bits each (an infinity or NaN is t[0] alone).
__device__ __forceinline__ void split3(const float (&x)[8], bf16x8 (&t)[3])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = __uint_as_float(__float_as_uint(x[i]) & 0xFFFF0000u);
        const float r = __builtin_isinf(x[i]) ? 0.0f : x[i] - a;
        const float b = __uint_as_float(__float_as_uint(r) & 0xFFFF0000u);
        t[0][i] = (__bf16)a;
        t[1][i] = (__bf16)b;
        t[2][i] = (__bf16)(r - b);
    }
}

// Adds the products of one step to a group's sums: acc[channel] and xs, the sum of x.
template <int XT>
struct Sums {
    v4f acc, xs;
};
template <>
struct Sums<DSQ_T_I8> {
    v4i acc, xs;
};

template <int XT>
__device__ __forceinline__ void step(uint32_t w, const Frag<XT> &x, Sums<XT> &s)
{
    if constexpr (XT == DSQ_T_BF16) {
        const bf16x8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
        s.acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_bf16(w), x.v, s.acc, 0, 0, 0);
        s.xs = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, x.v, s.xs, 0, 0, 0);
    } else if constexpr (XT == DSQ_T_F16) {
        const f16x8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
        s.acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_f16(w), x.v, s.acc, 0, 0, 0);
        s.xs = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, x.v, s.xs, 0, 0, 0);
    } else if constexpr (XT == DSQ_T_F32) {
        const bf16x8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
        bf16x8 t[3];
        split3(x.v, t);
        const bf16x8 c = codes_bf16(w);
#pragma unroll
        for (int i = 2; i >= 0; --i) {
            s.acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c, t[i], s.acc, 0, 0, 0);
            s.xs = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, t[i], s.xs, 0, 0, 0);
        }
    } else {
        s.acc = __builtin_amdgcn_mfma_i32_16x16x32_i8(codes_i8(w), x.v, s.acc, 0, 0, 0);
        s.xs = __builtin_amdgcn_mfma_i32_16x16x32_i8(0x0101010101010101L, x.v, s.xs, 0, 0, 0);
    }
}

__device__ __forceinline__ float load_out(const void *p, int64_t i, int type)
{
    return type == DSQ_T_F32 ? ((const float *)p)[i] : type == DSQ_T_F16 ? (float)((const _Float16 *)p)[i] : (float)((const __bf16 *)p)[i];
}
__device__ __forceinline__ void store_out(void *p, int64_t i, int type, float v)
{
    if (type == DSQ_T_F32) ((float *)p)[i] = v;
    else if (type == DSQ_T_F16) ((_Float16 *)p)[i] = (_Float16)v;
    else ((__bf16 *)p)[i] = (__bf16)v;
}

// GPB: groups in a block of 128 channels.
template <int XT, int MT, int GPB>
__global__ __launch_bounds__(64 * ROWS_WAVES) void w4_rows_kernel(DsqW4Args a)
{
    constexpr int SPG = 4 / GPB;         // steps of a group
    __shared__ v4f part[ROWS_WAVES][MT][64];
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int nt = blockIdx.x;
    const int64_t m0 = (int64_t)blockIdx.y * 16 * MT;
    const int KB = dsq_w4_round(a.K) / 128, Gp = KB * GPB;
    const v4u *w = reinterpret_cast<const v4u *>(a.w) + (size_t)nt * KB * 64 + lane;
    const v4u *sc = reinterpret_cast<const v4u *>(a.scales) + (size_t)nt * Gp * 4 + q;
    const size_t e = XT == DSQ_T_F32 ? 4 : XT == DSQ_T_I8 ? 1 : 2;
    v4f sum[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) sum[i] = (v4f){0.f, 0.f, 0.f, 0.f};
    for (int b = wave; b < KB; b += ROWS_WAVES) {
        const v4u wv = w[(size_t)b * 64];
        v4u sv[GPB];
#pragma unroll
        for (int g = 0; g < GPB; ++g) sv[g] = sc[(size_t)(b * GPB + g) * 4];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int64_t m = m0 + 16 * i + r;
            const void *row = (const char *)a.x + m * a.x_stride * (int64_t)e;
            Frag<XT> f[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) f[t] = load_frag<XT>(row, 128 * b + 32 * t + 8 * q, a.K, m < a.M);
#pragma unroll
            for (int g = 0; g < GPB; ++g) {
                Sums<XT> s = {};
#pragma unroll
                for (int t = 0; t < SPG; ++t) step<XT>(wv[g * SPG + t], f[g * SPG + t], s);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float scale = __uint_as_float(sv[g][c] & ~15u), zero = (float)(sv[g][c] & 15u);
                    sum[i][c] = __builtin_fmaf(scale, __builtin_fmaf(-zero, (float)s.xs[c], (float)s.acc[c]), sum[i][c]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) part[wave][i][lane] = sum[i];
    __syncthreads();
    for (int i = wave; i < MT; i += ROWS_WAVES) {
        v4f v = part[0][i][lane];
#pragma unroll
        for (int p = 1; p < ROWS_WAVES; ++p) v += part[p][i][lane];
        const int64_t m = m0 + 16 * i + r;
        if (m >= a.M) continue;
        const float xs = XT == DSQ_T_I8 ? a.x_scale[m] : 1.0f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int n = 16 * nt + 4 * q + c;
            if (n >= a.N) continue;
            float o = XT == DSQ_T_I8 ? v[c] * xs : v[c];
            if (a.bias) o += load_out(a.bias, n, a.out_type);
            store_out(a.out, m * a.out_stride + n, a.out_type, o);
        }
    }
}

template <int XT, int MT>
hipError_t launch_rows(const DsqW4Args &a, hipStream_t stream)
{
    const dim3 grid((unsigned)((a.N + 15) / 16), (unsigned)((a.M + 16 * MT - 1) / (16 * MT)));
    if (a.group == 32) w4_rows_kernel<XT, MT, 4><<<grid, 64 * ROWS_WAVES, 0, stream>>>(a);
    else if (a.group == 64) w4_rows_kernel<XT, MT, 2><<<grid, 64 * ROWS_WAVES, 0, stream>>>(a);
    else w4_rows_kernel<XT, MT, 1><<<grid, 64 * ROWS_WAVES, 0, stream>>>(a);
    return hipGetLastError();
}

template <int XT>
hipError_t launch_of(const DsqW4Args &a, hipStream_t stream)
{
    return a.M <= 16 ? launch_rows<XT, 1>(a, stream) : a.M <= 32 ? launch_rows<XT, 2>(a, stream) : launch_rows<XT, 4>(a, stream);
}

}  // namespace

hipError_t dsq_launch_w4_linear(const DsqW4Args &a, hipStream_t stream)
{
    switch (a.x_type) {
    case DSQ_T_F32: return launch_of<DSQ_T_F32>(a, stream);
    case DSQ_T_F16: return launch_of<DSQ_T_F16>(a, stream);
    case DSQ_T_BF16: return launch_of<DSQ_T_BF16>(a, stream);
    }
    return launch_of<DSQ_T_I8>(a, stream);
}
