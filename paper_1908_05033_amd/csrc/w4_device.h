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

// (WHOLE: channels k..k+7 exist.  Callers branch on the block and not here: behind a branch at each load it would be waited for.
// A lane whose row does not exist keeps what `f` holds: rows of a matrix product do not meet.)
template <int XT, bool WHOLE>
__device__ __forceinline__ void load_frag(Frag<XT> &f, const void *row, int k, int K, bool live)
{
    if (!live) return;
    if constexpr (XT == DSQ_T_I8) {
        // (rows end with their pitch, a multiple of 128, and what lies behind K meets levels of 0)
        f.v = *reinterpret_cast<const long *>((const int8_t *)row + k);
    } else {
        typedef typename Element<XT>::type E;
        if constexpr (WHOLE) {
            const Side<E, 8> s = load_side<E, 8>((const E *)row + k);
#pragma unroll
            for (int i = 0; i < 8; ++i) f.v[i] = s.at[i];
        } else if (sizeof(E) == 2 && K >= 8) {
            // the row's last eight, moved down by as many as lie before k
            const int back = k + 8 - K, n = 16 * (back < 0 ? 0 : back > 8 ? 8 : back);
            const Side<uint64_t, 2> s = load_side<uint64_t, 2>((const uint64_t *)((const E *)row + (back > 0 ? K - 8 : k)));
            const uint64_t lo = s.at[0], hi = s.at[1];
            const uint64_t to[2] = {n == 0 ? lo : n < 64 ? lo >> n | hi << (64 - n) : n < 128 ? hi >> (n - 64) : 0,
                                    n < 64 ? hi >> n : 0};
            __builtin_memcpy(&f, to, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const E v = ((const E *)row)[k + i < K ? k + i : 0];
                f.v[i] = k + i < K ? v : (E)0.0f;
            }
        }
    }
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

// Binary32 numbers are multiplied by 2^24 before they are cut in parts and summed, and the sums of a row by 2^-24 at the end: the last
// part of a number lies up to 23 places below it, past the smallest bfloat16 number from 2^-110 on.  Scaled, every part of every
// number is a normal one.  (The sums reach their range from 2^93 on: see product_in_64_bits.)  A multiplication more for each number
// costs the kernel for a few rows, whose waves all cut their rows, 4 to 8 % (us, without / with: 4 x 25088 to 4096 31.8 / 34.3, 3 x 4100
// to 1000 8.0 / 8.4, 16 x 4096 to 4096 10.9 / 11.0), the others 0 to 2 %; forming what remains after a cut with the dot product
// instruction, one for two, is no faster.
constexpr float kUp = 0x1p24f, kDown = 0x1p-24f;
template <int XT>
__device__ __forceinline__ void scale_up(Frag<XT> &f)
{
    if constexpr (XT == DSQ_T_F32)
#pragma unroll
        for (int i = 0; i < 8; ++i) f.v[i] *= kUp;
}

// x = t[0] + t[1] + t[2] exactly, eight significant bits each, cut towards zero: the upper halves of x and of what remains, two
// numbers moved at a time.  (An infinity or a NaN leaves NaN in t[1] and t[2], and makes its row NaN.)
__device__ __forceinline__ void split3(const float (&x)[8], bf16x8 (&t)[3])
{
    uint32_t to[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = x[2 * i], b = x[2 * i + 1];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            to[k][i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
            a -= __uint_as_float(__float_as_uint(a) & 0xFFFF0000u);
            b -= __uint_as_float(__float_as_uint(b) & 0xFFFF0000u);
        }
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) __builtin_memcpy(&t[k], to[k], 16);
}

// The sum over 4, 8 or 16 lanes side by side, in each of them: lanes exchanged by one and by two, then halves and rows of 16 mirrored.
template <int CONTROL>
__device__ __forceinline__ float plus_lane(float v)
{
    return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CONTROL, 0xF, 0xF, true));
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v)
{
    v = plus_lane<0xB1>(v);
    v = plus_lane<0x4E>(v);
    if (LANES > 4) v = plus_lane<0x141>(v);
    if (LANES > 8) v = plus_lane<0x140>(v);
    return v;
}

// The sum of a lane's eight numbers.
template <int XT>
__device__ __forceinline__ float sum8(const Frag<XT> &f)
{
    float s = 0.0f;
    if constexpr (XT == DSQ_T_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s += f.v[i];
    } else if constexpr (XT == DSQ_T_I8) {
        const v2u v = __builtin_bit_cast(v2u, f.v);
        const uint32_t lo = v.x, hi = v.y;
        s = (float)__builtin_amdgcn_sdot4((int)lo, 0x01010101, __builtin_amdgcn_sdot4((int)hi, 0x01010101, 0, false), false);
    } else {
        const v4u x = __builtin_bit_cast(v4u, f.v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t pair = x[i];       // (a bit_cast of the vector's element itself takes element 0)
            if constexpr (XT == DSQ_T_BF16) {
                const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
                s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), ones, s, false);
            } else {
                const f16x2 ones = {(_Float16)1.0f, (_Float16)1.0f};
                s = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, pair), ones, s, false);
            }
        }
    }
    return s;
}

// Rows of bfloat16 and binary32 numbers reach as far as the binary32 sums do: a group's sum of codes times x, or of x, may pass
// 2^128 where the result does not, and then the result is an infinity or a NaN.  Such results, and no others, are formed again
// from the levels in binary64, which no such sum overflows: output n of row m, by the lane that stores it.  Slow, and rare: 4096 to
// 4096 channels, bfloat16, 1024 rows of numbers around 1e37 take 12 ms (ordinary ones 43 us), one such row 0.35 ms.  A row that holds an
// infinity or a NaN ends at the first (all NaN: 95 us).
template <int XT>
constexpr bool kSumsOverflow = XT == DSQ_T_BF16 || XT == DSQ_T_F32;
__device__ __forceinline__ bool overflowed(float sum) { return !(__builtin_fabsf(sum) <= 3.402823466e38f); }
// Its arguments are the kernel's first, read again from where they were passed: kept for it, they cost scalar registers everywhere
// (one row, 4096 to 4096: 4.5 us with, 4.4 without).
template <int XT>
__device__ __forceinline__ float product_in_64_bits(int64_t m, int n)
{
    typedef typename Element<XT>::type E;
    typedef const __attribute__((address_space(4))) DsqW4Args *Passed;
    Passed passed = (Passed)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(passed));
    const struct {
        const void *x;
        int64_t x_stride;
        const uint32_t *w, *scales;
        int K, group;
    } a = {passed->x, passed->x_stride, passed->w, passed->scales, passed->K, passed->group};
    const int KB = dsq_w4_round(a.K) / 128, Gp = KB * (128 / a.group);
    const E *x = (const E *)a.x + m * a.x_stride;
    const uint32_t *w = a.w + (size_t)(n / 16) * KB * 256 + n % 16 * 4, *sc = a.scales + (size_t)(n / 16) * Gp * 16 + n % 16;
    double sum = 0.0;
    for (int k = 0; k < a.K; k += 8) {
        const uint32_t word = w[(size_t)(k / 128) * 256 + k % 32 * 8 + k % 128 / 32], s = sc[(size_t)(k / a.group) * 16];
        const double scale = (double)__uint_as_float(s & ~15u);
        const int zero = (int)(s & 15u);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int code = (int)(word >> (8 * (i & 3) + 4 * (i >> 2)) & 15u);
            if (k + i < a.K) sum += scale * (double)(code - zero) * (double)(float)x[k + i];
        }
        if (!(__builtin_fabs(sum) <= 1.7e308)) break;
    }
    return (float)sum;
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
