// Device-side helpers of the products with group-scaled 4-bit weights (gfx950 only).
#pragma once
#include "lm_device.h"

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef int v4i __attribute__((ext_vector_type(4)));

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

// (WHOLE: channels k..k+7 exist.  Callers branch on the block and not here: behind a branch at each load it would be waited for.)
template <int XT, bool WHOLE>
__device__ __forceinline__ Frag<XT> load_frag(const void *row, int k, int K, bool live)
{
    Frag<XT> f = {};
    if constexpr (XT == DSQ_T_I8) {
        // (rows end with their pitch, a multiple of 128, and what lies behind K meets levels of 0)
        if (live) f.v = *reinterpret_cast<const long *>((const int8_t *)row + k);
    } else {
        typedef typename Element<XT>::type E;
        const E *p = (const E *)row + k;
        if constexpr (WHOLE) {
            if (live) {
                const Side<E, 8> s = load_side<E, 8>(p);
#pragma unroll
                for (int i = 0; i < 8; ++i) f.v[i] = s.at[i];
            }
        } else if (live) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const E v = ((const E *)row)[k + i < K ? k + i : K - 1];
                f.v[i] = k + i < K ? v : (E)0.0f;
            }
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

// Adds the products of one step to a group's sums over a lane's four rows: acc for its output channel, xs those of x alone.
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
        s.acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v, codes_bf16(w), s.acc, 0, 0, 0);
        s.xs = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v, ones, s.xs, 0, 0, 0);
    } else if constexpr (XT == DSQ_T_F16) {
        const f16x8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
        s.acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(x.v, codes_f16(w), s.acc, 0, 0, 0);
        s.xs = __builtin_amdgcn_mfma_f32_16x16x32_f16(x.v, ones, s.xs, 0, 0, 0);
    } else if constexpr (XT == DSQ_T_F32) {
        const bf16x8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
        bf16x8 t[3];
        split3(x.v, t);
        const bf16x8 c = codes_bf16(w);
#pragma unroll
        for (int i = 2; i >= 0; --i) {
            s.acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t[i], c, s.acc, 0, 0, 0);
            s.xs = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t[i], ones, s.xs, 0, 0, 0);
        }
    } else {
        s.acc = __builtin_amdgcn_mfma_i32_16x16x32_i8(x.v, codes_i8(w), s.acc, 0, 0, 0);
        s.xs = __builtin_amdgcn_mfma_i32_16x16x32_i8(x.v, 0x0101010101010101L, s.xs, 0, 0, 0);
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
