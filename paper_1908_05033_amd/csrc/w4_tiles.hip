// Many rows times group-scaled 4-bit weights: a tiled product on the 32x32 matrix instructions; the choice of kernel and tile.
//
// A workgroup of eight waves owns 32 * MT rows x 32 * WN output channels.  Blocks of 128 input channels of its rows go through
// LDS (rows padded by 16 bytes: reads of a column of 16-byte units are free of bank conflicts); a wave takes 32 output
// channels, whose codes come from global memory in lane order, and all rows, so that a code is unpacked once for 32 * MT rows;
// WK waves share a channel's input blocks and join their sums in LDS at the end.  With the rows as the first operand a lane
// holds one output channel: its scale and zero point are one word a group.
//
// 8-bit rows: the operand is code - z as bytes, a group's sum an exact integer, converted and scaled once a group (two
// vector instructions an element, which no matrix instruction can take over).  Floats: the operand is the code, and the group's
// sum of x, from the staging of the rows, carries the zero point.
//
// Measured at K = 4096 and groups of 128: 2048 rows to 8192 channels 99 us (1.39 POP/s) with 8-bit rows, 156 us (0.88 PFLOP/s)
// with bfloat16 ones.  Of the former the vector instructions (15 for a matrix instruction: the scaling of the groups 8, the
// unpacking 4) fill 60 and the matrix instructions 30 of a compute unit's time; with two waves on a SIMD they overlap in part.
// 256 rows to 4096: 12 and 21 us.  Of the latter a call without work is 6, and for its 16 million codes the loads alone, the writes to
// LDS alone and the multiplication alone would take 8, 4 and 10: with one workgroup on a compute unit they too overlap in part.
#include <type_traits>

#include "w4_device.h"
#include "w4_plan.h"

namespace {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v16i __attribute__((ext_vector_type(16)));

template <int XT>
struct Tile {
    static constexpr int ES = sizeof(typename Element<XT>::type);
    static constexpr int PLANES = XT == DSQ_T_F32 ? 3 : 1;            // a binary32 number lies in LDS as its three parts
    static constexpr int PLANE = XT == DSQ_T_I8 ? 128 : 256;          // bytes of a plane of a block's row in LDS
    static constexpr int PITCH = PLANES * PLANE + 16;
    static constexpr int UNITS = PLANE / 16, CH = 128 / UNITS;        // units of a row that a thread stages, channels of one
    static constexpr int WORDS = CH * ES / 16;                        // 16-byte words of a unit in memory
};

// Code - zero of a word's eight codes as bytes: 128 + code - zero is between 113 and 143, without carries from byte to byte.
__device__ __forceinline__ void levels_i8(uint32_t w, uint32_t plus, int &lo, int &hi)
{
    lo = (int)(((w & 0x0F0F0F0Fu) + plus) ^ 0x80808080u);
    hi = (int)((((w >> 4) & 0x0F0F0F0Fu) + plus) ^ 0x80808080u);
}

// MT: tiles of 32 rows; WN x WK waves: 32 output channels each, and the WK-th part of an iteration's blocks, BPI each (fewer
// barriers: 3 % at 128 x 256); GPB: groups of a block.
template <int XT, int MT, int WN, int WK, int BPI, int GPB>
__global__ __launch_bounds__(64 * WN * WK, 2) void w4_tiles_kernel(DsqW4Args a, int tiles_m, int total, int xcd_chunk)
{
    typedef Tile<XT> L;
    constexpr bool INT = XT == DSQ_T_I8;
    constexpr int SPG = 4 / GPB;                                      // steps of 32 channels in a group
    constexpr int THREADS = 64 * WN * WK, ROWS = 32 * MT, BLOCK = ROWS * L::PITCH;
    constexpr int STEP = WK * BPI;                                    // blocks of an iteration
    constexpr bool DEEP = BPI == 1;                                   // rows are fetched two iterations ahead
    constexpr int LOADS = ROWS * L::UNITS * STEP / THREADS;           // units a thread stages
    constexpr int XSUM = INT ? 0 : GPB * ROWS;                        // sums of x of a block's groups
    extern __shared__ __attribute__((aligned(16))) char lds[];       // [2][STEP] blocks, then [2][STEP] sums
    float *xsums = reinterpret_cast<float *>(lds + 2 * STEP * BLOCK);

    // Workgroups are dealt to the 8 XCDs in turn: each gets a contiguous range of tiles, the row tiles of one channel tile
    // together, so that its weights are read into one L2 only
    const int logical = ((int)blockIdx.x & 7) * xcd_chunk + ((int)blockIdx.x >> 3);
    if (logical >= total) return;
    const int nt = logical / tiles_m;
    const int64_t m0 = (int64_t)(logical - nt * tiles_m) * ROWS;
    const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wn = wave % WN, wk = wave / WN;
    const int KB = dsq_w4_round(a.K) / 128, Gp = KB * GPB, iters = (KB + STEP - 1) / STEP;
    const int n0 = nt * 32 * WN + 32 * wn;
    // this lane's channel: 16-channel block (r / 16), column r % 16; its halves of 16 input channels
    const size_t ct = (size_t)w4_channel_tile(a.N, n0, r);
    const v4u *w = reinterpret_cast<const v4u *>(a.w) + ct * KB * 64 + 32 * h + r % 16;
    const uint32_t *sc = a.scales + ct * Gp * 16 + r % 16;

    v16f sum[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int c = 0; c < 16; ++c) sum[i][c] = 0.0f;

    const int unit = threadIdx.x % L::UNITS, line0 = threadIdx.x / L::UNITS;
    constexpr int LINES = THREADS / L::UNITS;                         // rows a load instruction of the workgroup covers
    typedef Side<v4u, L::WORDS> Unit;
    Unit xa[LOADS], xb[LOADS];
    auto load_rows = [&](int it, Unit (&xr)[LOADS]) __attribute__((always_inline)) {
        // (8-bit rows without a branch around the loads: where it next waits for a scale the compiler would wait for them too, 107 us
        // for 98 at 2048 x 4096 to 8192.  Floats win nothing by it, and lose what the loads past the end take.)
        if (!INT && it >= iters) {                                    // (meets scales of 0: any number will do)
#pragma unroll
            for (int j = 0; j < LOADS; ++j)
#pragma unroll
                for (int k = 0; k < L::WORDS; ++k) xr[j].at[k] = (v4u){0u, 0u, 0u, 0u};
            return;
        }
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int line = line0 + j * LINES, row = line % ROWS, at = it * STEP + line / ROWS;
            int64_t m = m0 + row;
            m = m < a.M ? m : a.M - 1;                                // (past the end: loaded and not stored)
            // past the last block floats of that one again, as its weights: what overflows under scales of 0 has done so before.  Past
            // the row's end its last unit: of levels or scales of 0 (8-bit rows), or cut off by `cut`.
            const int b = INT ? at : min(at, KB - 1);
            const int k = 128 * b + L::CH * unit, last = (INT ? 128 * KB : a.K) - L::CH;
            xr[j] = load_side<v4u, L::WORDS>((const v4u *)((const char *)a.x + (m * a.x_stride + (k < last ? k : last)) * L::ES));
        }
    };
    // Floats of the last blocks, k..k+7 of a row of K: moved down by as many as lie before k, zeros behind K.
    auto cut = [&](Unit &x, int k) __attribute__((always_inline)) {
        const int back = k + 8 - a.K;
        if constexpr (XT == DSQ_T_F32) {
            float at[8];
            __builtin_memcpy(at, &x, 32);
#pragma unroll
            for (int by = 1; by < 8; by *= 2)
#pragma unroll
                for (int i = 0; i < 8; ++i) at[i] = back <= 0 || !(back & by) ? at[i] : i + by < 8 ? at[i + by] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) at[i] = back < 8 ? at[i] : 0.0f;
            __builtin_memcpy(&x, at, 32);
        } else {
            const int n = 16 * (back < 0 ? 0 : back > 8 ? 8 : back);
            uint64_t at[2];
            __builtin_memcpy(at, &x, 16);
            const uint64_t lo = n >= 128 ? 0 : n >= 64 ? at[1] : at[0], hi = n >= 64 ? 0 : at[1];
            const uint64_t to[2] = {lo >> (n & 63) | hi << 1 << (63 - (n & 63)), hi >> (n & 63)};
            __builtin_memcpy(&x, to, 16);
        }
    };
    const int it_cut = !INT && a.K % 128 ? iters - 1 : -1;
    auto store_rows = [&](int to, int it, Unit (&xr)[LOADS]) __attribute__((always_inline)) {
        if constexpr (!INT)
            if (it == it_cut)
#pragma unroll
                for (int j = 0; j < LOADS; ++j) {
                    cut(xr[j], 128 * (it * STEP + (line0 + j * LINES) / ROWS) + 8 * unit);
                    __builtin_amdgcn_sched_barrier(0);                // (one after the other: side by side they spill)
                }
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int line = line0 + j * LINES, row = line % ROWS, k = line / ROWS;
            v4u *at = reinterpret_cast<v4u *>(lds + (to * STEP + k) * BLOCK + row * L::PITCH + 16 * unit);
            if constexpr (INT) {
                *at = xr[j].at[0];
            } else {
                Frag<XT> f;
                __builtin_memcpy(&f, &xr[j], sizeof f);
                scale_up(f);
                if constexpr (XT == DSQ_T_F32) {
                    bf16x8 t[3];
                    split3(f.v, t);
#pragma unroll
                    for (int i = 0; i < 3; ++i) at[i * L::PLANE / 16] = __builtin_bit_cast(v4u, t[i]);
                } else {
                    *at = xr[j].at[0];
                }
                // the sum of a group of x: eight channels a lane, 4 * SPG lanes side by side
                float s = sum8(f);
                s = lanes_sum<4 * SPG>(s);
                if (unit % (4 * SPG) == 0) xsums[(to * STEP + k) * XSUM + unit / (4 * SPG) * ROWS + row] = s;
            }
        }
    };
    auto load_weights = [&](int it, v4u (&to)[BPI][2], uint32_t (&s)[BPI][GPB]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < BPI; ++j) {
            // (past the end: the last block's with scales of 0)
            const int at = it * STEP + wk * BPI + j;
            const bool live = it < iters && at < KB;
            const int b = live ? at : KB - 1;
            to[j][0] = w[(size_t)b * 64];
            to[j][1] = w[(size_t)b * 64 + 16];
#pragma unroll
            for (int g = 0; g < GPB; ++g) {
                s[j][g] = sc[(size_t)(b * GPB + g) * 16];
                if (!live) s[j][g] = 0;
            }
        }
    };
    // One block of input channels from LDS block `at`.
    auto block = [&](int at, const v4u (&wv)[2], const uint32_t (&sv)[GPB]) __attribute__((always_inline)) {
        const char *base = lds + at * BLOCK + r * L::PITCH + (INT ? 16 : 32) * h;
        const float *xsum = xsums + at * XSUM;
        // Units of one group and 32 rows: the matrix instructions of a unit stand beside the scaling of the one before, and its
        // rows are read from LDS one unit ahead.  (Left to itself the compiler reads the rows of all units first and spills, or
        // reads each operand right before its instruction and waits.)
        constexpr int XF = INT ? SPG : 2 * SPG * L::PLANES;           // operands of a unit's rows
        constexpr int PART = XF < 4 ? XF : L::PLANES == 3 ? 6 : 4, PARTS = XF / PART;      // ... of which so many are read ahead
        v4i xf[2][PART];
        v16f facc[2];
        v16i iacc[2];
        v4i lev[SPG];
        auto read_rows = [&](int p) __attribute__((always_inline)) {
            const int g = p / PARTS / MT, i = p / PARTS % MT;
#pragma unroll
            for (int j = 0; j < PART; ++j) {
                const int o = p % PARTS * PART + j, t = o / L::PLANES;
                xf[p & 1][j] = *reinterpret_cast<const v4i *>(base + 32 * i * L::PITCH + (INT ? 32 * (g * SPG + t) : 64 * (g * SPG + t / 2) + 16 * (t % 2)) + L::PLANE * (o % L::PLANES));
            }
        };
        auto scaled = [&](int u) __attribute__((always_inline)) {
            const int g = u / MT, i = u % MT;
            const float scale = __uint_as_float(sv[g] & ~15u);
            if constexpr (INT) {
#pragma unroll
                for (int c = 0; c < 16; ++c) sum[i][c] = __builtin_fmaf(scale, (float)iacc[u & 1][c], sum[i][c]);
            } else {
                const float shift = -scale * (float)(sv[g] & 15u);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const v4f xs = *reinterpret_cast<const v4f *>(xsum + g * ROWS + 32 * i + 8 * c + 4 * h);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        sum[i][4 * c + k] = __builtin_fmaf(shift, xs[k], __builtin_fmaf(scale, facc[u & 1][4 * c + k], sum[i][4 * c + k]));
                }
            }
            // (done here: the compiler would move the scaling of a whole block behind it, and spill the units' sums)
            asm volatile("" : "+v"(sum[i]));
        };
        read_rows(0);
#pragma unroll
        for (int p = 0; p < GPB * MT * PARTS; ++p) {
            const int u = p / PARTS, g = u / MT, i = u % MT;
            if (p + 1 < GPB * MT * PARTS) read_rows(p + 1);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (INT) {
                if (i == 0) {
                    const uint32_t plus = 0x80808080u - (sv[g] & 15u) * 0x01010101u;
#pragma unroll
                    for (int t = 0; t < SPG; ++t) {
                        int p0, p1, p2, p3;
                        levels_i8(wv[0][g * SPG + t], plus, p0, p1);
                        levels_i8(wv[1][g * SPG + t], plus, p2, p3);
                        lev[t] = (v4i){p0, p1, p2, p3};
                    }
                }
                v16i acc = {};
#pragma unroll
                for (int t = 0; t < SPG; ++t) acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(xf[p & 1][t], lev[t], acc, 0, 0, 0);
                iacc[u & 1] = acc;
            } else {
                v16f acc = {};
                if (p % PARTS) acc = facc[u & 1];
#pragma unroll
                for (int j = 0; j < PART; ++j) {
                    const int t = (p % PARTS * PART + j) / L::PLANES;
                    const v4i x = xf[p & 1][j];
                    const uint32_t codes = wv[t % 2][g * SPG + t / 2];
                    if constexpr (XT != DSQ_T_F16)
                        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), codes_bf16(codes), acc, 0, 0, 0);
                    else
                        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), codes_f16(codes), acc, 0, 0, 0);
                }
                facc[u & 1] = acc;
            }
            if (u > 0 && p % PARTS == 0) scaled(u - 1);
            if constexpr (INT)                                        // (a share of the scaling behind each matrix instruction)
#pragma unroll
                for (int t = 0; t < SPG; ++t) {
                    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x2, 32 / SPG, 0);
                }
            __builtin_amdgcn_sched_barrier(0);
        }
        scaled(GPB * MT - 1);
    };

    // Two sets of weight registers in turn (a copy of a prefetched set would wait for it), loaded again once their block is
    // multiplied; the rows of the next iteration, and of the one after it too where it is one block (bfloat16: 2 to 5 %), are
    // under way meanwhile.  The loop runs an even number of iterations: what is fetched past the end meets scales of 0.
    auto blocks = [&](int from, const v4u (&wv)[BPI][2], const uint32_t (&sv)[BPI][GPB]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < BPI; ++j) block(from * STEP + wk * BPI + j, wv[j], sv[j]);
    };
    v4u wa[BPI][2], wb[BPI][2];
    uint32_t sa[BPI][GPB], sb[BPI][GPB];
    load_rows(0, xa);
    load_weights(0, wa, sa);
    if (DEEP) load_rows(1, xb);
    load_weights(1, wb, sb);
    store_rows(0, 0, xa);
    __syncthreads();
    for (int it = 0; it < iters; it += 2) {
        load_rows(it + (DEEP ? 2 : 1), xa);
        __builtin_amdgcn_sched_barrier(0);
        blocks(0, wa, sa);
        load_weights(it + 2, wa, sa);
        store_rows(1, it + 1, DEEP ? xb : xa);
        __syncthreads();
        load_rows(it + (DEEP ? 3 : 2), xb);
        __builtin_amdgcn_sched_barrier(0);
        blocks(1, wb, sb);
        load_weights(it + 3, wb, sb);
        store_rows(0, it + 2, DEEP ? xa : xb);
        __syncthreads();
    }
    // Registers 4q..4q+3 of a lane are rows 8q + 4h + 0..3 of a tile of 32: the WK waves of a channel tile leave their sums in
    // LDS, and each joins and stores the quarters q of its own.
    v4f *part = reinterpret_cast<v4f *>(lds);                         // [wave][row tile][quarter][lane]
    if constexpr (WK > 1) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                part[((wave * MT + i) * 4 + q) * 64 + lane] = (v4f){sum[i][4 * q], sum[i][4 * q + 1], sum[i][4 * q + 2], sum[i][4 * q + 3]};
        __syncthreads();
    }
    const int n = n0 + r;
    if (n >= a.N) return;
    constexpr int QS = 4 / WK;                                        // quarters of a tile that a wave stores
    auto store = [&](auto type) __attribute__((always_inline)) {
        typedef decltype(type) E;
        const float bias = a.bias ? (float)((const E *)a.bias)[n] : 0.0f;
        float mark = 0.0f;                                            // NaN once a sum has overflowed
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int64_t m = m0 + 32 * i + 8 * wk + 4 * h;           // the lane's first row of the tile
            const int live = a.M - m < 32 ? (int)(a.M - m) : 32;
            if (live <= 0) break;
            float scale[4 * QS];
            if constexpr (INT)
#pragma unroll
                for (int c = 0; c < 4 * QS; ++c) {
                    const int at = 8 * WK * (c / 4) + c % 4;
                    scale[c] = a.x_scale[m + (at < live ? at : 0)];
                }
            E *out = (E *)a.out + m * a.out_stride + n;
#pragma unroll
            for (int j = 0; j < QS; ++j) {
                v4f s;
                if constexpr (WK > 1) {
                    const int q = j * WK + wk;
                    s = part[((wn * MT + i) * 4 + q) * 64 + lane];
#pragma unroll
                    for (int k = 1; k < WK; ++k) s += part[(((k * WN + wn) * MT + i) * 4 + q) * 64 + lane];
                } else {
                    s = (v4f){sum[i][4 * j], sum[i][4 * j + 1], sum[i][4 * j + 2], sum[i][4 * j + 3]};
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float o = INT ? s[c] * scale[4 * j + c] : XT == DSQ_T_F32 ? s[c] * kDown : s[c];
                    if (a.bias) o += bias;
                    if (kSumsOverflow<XT>) mark = __builtin_fmaf(s[c], 0.0f, mark);
                    if (8 * WK * j + c < live) out[(8 * WK * j + c) * a.out_stride] = (E)o;
                }
            }
        }
        if constexpr (kSumsOverflow<XT>)
            if (__builtin_expect(mark != 0.0f, 0))                    // (the lane looks through what it has stored)
                for (int e = 0; e < 4 * QS * MT; ++e) {
                    const int64_t m = m0 + 32 * (e / (4 * QS)) + 8 * wk + 4 * h + 8 * WK * (e / 4 % QS) + e % 4;
                    if (m >= a.M) break;
                    E *out = (E *)a.out + m * a.out_stride + n;
                    if (!overflowed((float)*out)) continue;
                    float o = product_in_64_bits<XT>(m, n);
                    if (a.bias) o += bias;
                    *out = (E)o;
                }
    };
    if constexpr (!INT) store((typename Element<INT ? DSQ_T_F32 : XT>::type)0.0f);
    else if (a.out_type == DSQ_T_BF16) store((__bf16)0.0f);
    else if (a.out_type == DSQ_T_F16) store((_Float16)0.0f);
    else store(0.0f);
}

template <int XT, int MT, int WN, int WK, int BPI, int GPB>
hipError_t launch_of(const DsqW4Args &a, hipStream_t stream)
{
    typedef Tile<XT> L;
    constexpr int STAGE = 2 * WK * BPI * (32 * MT * L::PITCH + (XT == DSQ_T_I8 ? 0 : GPB * 32 * MT * 4));
    constexpr int JOIN = WK > 1 ? WN * WK * MT * 64 * 64 : 0, LDS = STAGE > JOIN ? STAGE : JOIN;
    const int64_t tiles_m = ((int64_t)a.M + 32 * MT - 1) / (32 * MT), tiles_n = ((int64_t)a.N + 32 * WN - 1) / (32 * WN);
    const int64_t total = tiles_m * tiles_n, xcd_chunk = (total + 7) / 8;
    if (xcd_chunk * 8 * 64 * WN * WK >= 1LL << 32) return hipErrorInvalidConfiguration;
    auto kern = w4_tiles_kernel<XT, MT, WN, WK, BPI, GPB>;
    if (LDS > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
        if (e != hipSuccess) return e;
    }
    kern<<<(unsigned)(8 * xcd_chunk), 64 * WN * WK, LDS, stream>>>(a, (int)tiles_m, (int)total, (int)xcd_chunk);
    return hipGetLastError();
}

template <int XT, int MT, int WN, int WK, int BPI = 1>
hipError_t launch_groups(const DsqW4Args &a, hipStream_t stream)
{
    return a.group == 32 ? launch_of<XT, MT, WN, WK, BPI, 4>(a, stream)
           : a.group == 64 ? launch_of<XT, MT, WN, WK, BPI, 2>(a, stream) : launch_of<XT, MT, WN, WK, BPI, 1>(a, stream);
}

template <int XT>
hipError_t launch_tiles(const DsqW4Args &a, hipStream_t stream)
{
    constexpr bool INT = XT == DSQ_T_I8;
    switch (w4_least_time(a.M, a.N, INT ? kW4Codes : kW4Half)) {
    case 0: return launch_groups<XT, 1, 2, 4>(a, stream);
    case 1: return launch_groups<XT, 2, 2, 4>(a, stream);
    case 2: return launch_groups<XT, 2, 4, 2>(a, stream);
    case 3: return launch_groups<XT, 2, 8, 1, 2>(a, stream);
    default: return launch_groups<XT, 4, 8, 1, INT ? 2 : 1>(a, stream);       // (floats: two blocks an iteration would spill)
    }
}

hipError_t launch_f32(const DsqW4Args &a, hipStream_t stream)
{
    switch (a.K < 8 ? 0 : w4_least_time(a.M, a.N, kW4Single)) {       // (the tiles take eight channels of a row at a time)
    case 0: return dsq_launch_w4_rows(a, stream);
    case 1: return launch_groups<DSQ_T_F32, 1, 4, 2>(a, stream);
    case 2: return launch_groups<DSQ_T_F32, 1, 8, 1>(a, stream);
    default: return launch_groups<DSQ_T_F32, 2, 8, 1>(a, stream);
    }
}

}  // namespace

hipError_t dsq_launch_w4_linear(const DsqW4Args &a, hipStream_t stream)
{
    if (a.M == 1) return dsq_launch_w4_row(a, stream);
    if (a.x_type == DSQ_T_F32) return launch_f32(a, stream);
    if (a.x_type == DSQ_T_I8) return a.M <= 16 ? dsq_launch_w4_rows(a, stream) : launch_tiles<DSQ_T_I8>(a, stream);
    // (as above: the tiles take eight channels of a row at a time)
    if (a.M <= 16 || a.K < 8) return dsq_launch_w4_rows(a, stream);
    return a.x_type == DSQ_T_F16 ? launch_tiles<DSQ_T_F16>(a, stream) : launch_tiles<DSQ_T_BF16>(a, stream);
}
