// A few rows times group-scaled 4-bit weights.
//
// As in w4_row.hip a wave owns output channels and a share of the blocks of 128 input channels; the waves of a workgroup
// join their sums in LDS, in a fixed order.  Each wave reads the rows of its blocks straight into the operands' registers: its
// share of them is read by no other wave of the workgroup, so LDS would only add barriers.  A matrix product with ones gives the
// group's sum of x for the zero points.  Two sets of registers in turn: while one is multiplied the other is under way.
//
// Bound by the codes' way from memory and, in calls this short, by the tail of one round of workgroups: 4 float16 rows, 25088 to
// 4096 channels in groups of 64, 15.3 us (3.8 TB/s); 16 8-bit rows, 4096 to 12288 in groups of 128, 8.6 us (3.1 TB/s).
#include "w4_device.h"

namespace {

constexpr int WAVES = 8;

// Adds the products of one step to a group's sums over a lane's four rows: acc for its output channels, xs those of x alone.
template <int XT>
struct Acc {
    typedef v4f type;
};
template <>
struct Acc<DSQ_T_I8> {
    typedef v4i type;
};
template <int XT, int NT>
__device__ __forceinline__ void step(const uint32_t (&w)[NT], const Frag<XT> &x, typename Acc<XT>::type (&acc)[NT], typename Acc<XT>::type &xs)
{
    if constexpr (XT == DSQ_T_BF16) {
        const bf16x8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v, codes_bf16(w[n]), acc[n], 0, 0, 0);
        xs = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.v, ones, xs, 0, 0, 0);
    } else if constexpr (XT == DSQ_T_F16) {
        const f16x8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x.v, codes_f16(w[n]), acc[n], 0, 0, 0);
        xs = __builtin_amdgcn_mfma_f32_16x16x32_f16(x.v, ones, xs, 0, 0, 0);
    } else if constexpr (XT == DSQ_T_F32) {
        const bf16x8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
        bf16x8 t[3], c[NT];
        Frag<XT> up = x;
        scale_up(up);
        split3(up.v, t);
#pragma unroll
        for (int n = 0; n < NT; ++n) c[n] = codes_bf16(w[n]);
#pragma unroll
        for (int i = 2; i >= 0; --i) {
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t[i], c[n], acc[n], 0, 0, 0);
            xs = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t[i], ones, xs, 0, 0, 0);
        }
    } else {
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n] = __builtin_amdgcn_mfma_i32_16x16x32_i8(x.v, codes_i8(w[n]), acc[n], 0, 0, 0);
        xs = __builtin_amdgcn_mfma_i32_16x16x32_i8(x.v, 0x0101010101010101L, xs, 0, 0, 0);
    }
}

// NT: tiles of 16 output channels a wave owns; CHUNK: blocks of a set of registers; GPB: groups of a block.
template <int XT, int NT, int CHUNK, int GPB>
__global__ __launch_bounds__(64 * WAVES) void w4_rows_kernel(DsqW4Args a)
{
    constexpr int SPG = 4 / GPB;                    // steps of a group
    __shared__ v4f part[WAVES][NT][64];
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t m0 = (int64_t)blockIdx.y * 16;
    const int KB = dsq_w4_round(a.K) / 128, Gp = KB * GPB;
    // (the packed channels are rounded up to 128: every tile of a wave is there)
    const v4u *w = reinterpret_cast<const v4u *>(a.w) + (size_t)blockIdx.x * NT * KB * 64;
    const uint32_t *sc = a.scales + (size_t)blockIdx.x * NT * Gp * 16;
    constexpr int64_t e = sizeof(typename Element<XT>::type);
    const char *row = (const char *)a.x + ((m0 + r) * a.x_stride + 8 * q) * e;
    const bool live = m0 + r < a.M;
    v4f sum[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) sum[n] = (v4f){0.f, 0.f, 0.f, 0.f};

    struct Set {
        v4u w[CHUNK][NT];
        uint32_t s[CHUNK][NT][GPB];
        Frag<XT> x[CHUNK][4];
    } sa, sb;
    // (lanes without a row are never loaded: whatever they hold stays in rows that are not stored)
#pragma unroll
    for (int j = 0; j < CHUNK; ++j)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            Frag<XT> &fa = sa.x[j][t], &fb = sb.x[j][t];
            if constexpr (XT == DSQ_T_F32)
#pragma unroll
                for (int k = 0; k < 8; ++k) asm volatile("" : "=v"(fa.v[k]), "=v"(fb.v[k]));
            else asm volatile("" : "=v"(fa.v), "=v"(fb.v));
        }
    // whole blocks (8-bit rows have no others: they end with their pitch)
    const int whole = XT == DSQ_T_I8 ? KB : a.K / 128;
    auto load_weights = [&](int b, v4u (&wv)[NT], uint32_t (&sv)[NT][GPB]) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            wv[n] = w[((size_t)n * KB + b) * 64 + lane];
#pragma unroll
            for (int g = 0; g < GPB; ++g) sv[n][g] = sc[((size_t)n * Gp + b * GPB + g) * 16 + r];
        }
    };
    auto load = [&](int b0, Set &s) __attribute__((always_inline)) {
        if (b0 >= whole) return;
#pragma unroll
        for (int j = 0; j < CHUNK; ++j) load_weights(min(b0 + j * WAVES, whole - 1), s.w[j], s.s[j]);       // (past the end: loaded and not used)
#pragma unroll
        for (int j = 0; j < CHUNK; ++j)
#pragma unroll
            for (int t = 0; t < 4; ++t) load_frag<XT, true>(s.x[j][t], row, 128 * min(b0 + j * WAVES, whole - 1) + 32 * t, a.K, live);
    };
    auto block = [&](const v4u (&wv)[NT], const uint32_t (&sv)[NT][GPB], const Frag<XT> (&f)[4]) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < GPB; ++g) {
            typename Acc<XT>::type acc[NT] = {}, xs = {};
#pragma unroll
            for (int t = g * SPG; t < (g + 1) * SPG; ++t) {
                uint32_t words[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) words[n] = wv[n][t];
                step<XT, NT>(words, f[t], acc, xs);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float scale = __uint_as_float(sv[n][g] & ~15u), zero = (float)(sv[n][g] & 15u);
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    sum[n][c] = __builtin_fmaf(scale, __builtin_fmaf(-zero, (float)xs[c], (float)acc[n][c]), sum[n][c]);
            }
        }
    };
    auto multiply = [&](int b0, const Set &s) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < CHUNK; ++j)
            if (b0 + j * WAVES < whole) block(s.w[j], s.s[j], s.x[j]);
    };
    load(wave, sa);
    for (int b0 = wave; b0 < whole; b0 += 2 * WAVES * CHUNK) {
        load(b0 + WAVES * CHUNK, sb);
        multiply(b0, sa);
        load(b0 + 2 * WAVES * CHUNK, sa);
        multiply(b0 + WAVES * CHUNK, sb);
    }
    if (XT != DSQ_T_I8 && whole < KB && wave == whole % WAVES) {
        load_weights(whole, sa.w[0], sa.s[0]);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            load_frag<XT, false>(sa.x[0][t], row - 8 * q * e, 128 * whole + 32 * t + 8 * q, a.K, live);
            __builtin_amdgcn_sched_barrier(0);
        }
        block(sa.w[0], sa.s[0], sa.x[0]);
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) part[wave][i][lane] = sum[i];
    __syncthreads();
    for (int i = wave; i < NT; i += WAVES) {
        v4f v = part[0][i][lane];
#pragma unroll
        for (int p = 1; p < WAVES; ++p) v += part[p][i][lane];
        const int n = 16 * ((int)blockIdx.x * NT + i) + r;
        if (n >= a.N) continue;
        const float bias = a.bias ? load_out(a.bias, n, a.out_type) : 0.0f;
        uint32_t again = 0;                         // results to be formed again
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int64_t m = m0 + 4 * q + c;
            if (m >= a.M) continue;
            if (kSumsOverflow<XT>) again |= overflowed(v[c]) ? 1u << c : 0u;
            float o = XT == DSQ_T_I8 ? v[c] * a.x_scale[m] : XT == DSQ_T_F32 ? v[c] * kDown : v[c];
            if (a.bias) o += bias;
            store_out(a.out, m * a.out_stride + n, a.out_type, o);
        }
        if constexpr (kSumsOverflow<XT>)
            for (; again; again &= again - 1) {
                const int64_t m = m0 + 4 * q + __builtin_ctz(again);
                float o = product_in_64_bits<XT>(m, n);
                if (a.bias) o += bias;
                store_out(a.out, m * a.out_stride + n, a.out_type, o);
            }
    }
}

template <int XT, int NT, int CHUNK>
hipError_t launch_rows(DsqW4Args a, hipStream_t stream)
{
    const int64_t tiles_n = ((int64_t)a.N + 16 * NT - 1) / (16 * NT), out_size = a.out_type == DSQ_T_F32 ? 4 : 2;
    // (a launch holds under 2^32 threads and 2^16 workgroups in its second dimension)
    const int most = (int)((1 << 22) / tiles_n < 32768 ? (1 << 22) / tiles_n : 32768) * 16;
    for (int left = a.M; left > 0; left -= most) {
        a.M = left < most ? left : most;
        const dim3 grid((unsigned)tiles_n, (unsigned)((a.M + 15) / 16));
        if (a.group == 32) w4_rows_kernel<XT, NT, CHUNK, 4><<<grid, 64 * WAVES, 0, stream>>>(a);
        else if (a.group == 64) w4_rows_kernel<XT, NT, CHUNK, 2><<<grid, 64 * WAVES, 0, stream>>>(a);
        else w4_rows_kernel<XT, NT, CHUNK, 1><<<grid, 64 * WAVES, 0, stream>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        a.x = (const char *)a.x + most * a.x_stride * (int64_t)sizeof(typename Element<XT>::type);
        a.out = (char *)a.out + most * a.out_stride * out_size;
        if (XT == DSQ_T_I8) a.x_scale += most;
    }
    return hipSuccess;
}

template <int XT>
hipError_t launch_of(const DsqW4Args &a, hipStream_t stream)
{
    // (binary32 rows take twice the registers: 16 x 4096 -> 4096 12.5 us with one tile a wave, 13.0 with two)
    if constexpr (XT == DSQ_T_F32) return launch_rows<XT, 1, 1>(a, stream);
    else {
        // A wave that owns more channels reads the rows less often and leaves fewer waves (us, 1 / 2 / 4 tiles a wave:
        // 4 x 25088 -> 4096 18.6 / 23.5 / 34.1, 4 x 8192 -> 5120 11.8 / 9.6 / 12.7, 8 x 8192 -> 8192 15.2 / 11.8 / 14.6,
        // 8 x 8192 -> 10240 20.7 / 17.6 / 13.9, 16 x 4096 -> 12288 16.6 / 12.9 / 10.7)
        const int64_t tiles = ((int64_t)a.N + 15) / 16;
        if (tiles >= 576) return launch_rows<XT, 4, 1>(a, stream);
        if (tiles >= 288) return launch_rows<XT, 2, 1>(a, stream);
        return launch_rows<XT, 1, 2>(a, stream);
    }
}

}  // namespace

hipError_t dsq_launch_w4_rows(const DsqW4Args &a, hipStream_t stream)
{
    switch (a.x_type) {
    case DSQ_T_F32: return launch_of<DSQ_T_F32>(a, stream);
    case DSQ_T_F16: return launch_of<DSQ_T_F16>(a, stream);
    case DSQ_T_BF16: return launch_of<DSQ_T_BF16>(a, stream);
    }
    return launch_of<DSQ_T_I8>(a, stream);
}
