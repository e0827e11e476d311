// One row times group-scaled 4-bit weights:  out[n] = sum over groups g of s[n][g] * sum over k in g of (code - z) x[k].
//
// The sum of a group runs on the 16x16x32 matrix instructions with exact operands: a code is converted to the type of
// x (a byte 0..15 is the e4m3 number code * 2^-9, which one instruction turns into bf16 or f16 times 2^9), binary32
// activations are cut into three bf16 terms, 8-bit rows meet the codes as bytes.  The zero point's share comes from the
// group's sum of x, formed once when the row is brought to LDS.  Groups are joined in binary32.
//
// Bound by the weights' way from memory: every code is read once.  A wave owns 16 output channels and every KS-th block of
// 128 input channels, 8 KB of codes under way; KS waves join their sums in LDS, in a fixed order.  The row lies in LDS, a
// segment of input channels at a time, shared by the workgroup's waves.  Fifteen of the sixteen rows of a matrix instruction go to
// waste; it still takes a quarter of the time that its codes take from memory.
//
// Measured with bfloat16 rows and groups of 128: 8192 to 32768 channels 28.2 us (5.1 TB/s), 4096 to 4096 4.1 us, a launch and one
// round of memory latency.
#include "w4_device.h"

namespace {

constexpr int WAVES = 8, CHUNK = 4;     // blocks of a set of weight registers

template <int XT>
struct Row {
    // bytes of a channel in LDS and the terms of one
    static constexpr int ES = XT == DSQ_T_I8 ? 1 : 2, TERMS = XT == DSQ_T_F32 ? 3 : 1;
};

// GPB: groups in a block of 128 channels.
template <int XT, int GPB>
__global__ __launch_bounds__(64 * WAVES) void w4_row_kernel(DsqW4Args a, int KS, int seg)
{
    typedef Row<XT> L;
    constexpr int SPG = 4 / GPB;                    // steps of a group
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int ks = wave % KS, tiles = (a.N + 15) / 16, mine = (int)blockIdx.x * (WAVES / KS) + wave / KS;
    const int nt = min(mine, tiles - 1);            // (a wave past the last tile repeats it and stores nothing)
    const int KB = dsq_w4_round(a.K) / 128, Gp = KB * GPB;
    const v4u *w = reinterpret_cast<const v4u *>(a.w) + (size_t)nt * KB * 64;
    const uint32_t *sc = a.scales + (size_t)nt * Gp * 16;
    const int plane = seg * 128 * L::ES;            // bytes of a term
    float *xsums = reinterpret_cast<float *>(lds + L::TERMS * plane);               // [seg * GPB]
    float sum = 0.0f;                               // lanes 0..15: the tile's channels (the others' are of rows that do not exist)

    auto load = [&](int j, v4u (&wv)[CHUNK], uint32_t (&sv)[CHUNK][GPB]) __attribute__((always_inline)) {
        if (ks + j * KS >= KB) return;
#pragma unroll
        for (int c = 0; c < CHUNK; ++c) {
            const int b = min(ks + (j + c) * KS, KB - 1);       // (past the end: loaded and not used)
            wv[c] = w[(size_t)b * 64 + lane];
#pragma unroll
            for (int g = 0; g < GPB; ++g) sv[c][g] = sc[(size_t)(b * GPB + g) * 16 + r];
        }
    };
    // Blocks j .. j + CHUNK - 1 of this wave; `first`: the segment's first block.
    auto chunk = [&](int j, int first, const v4u (&wv)[CHUNK], const uint32_t (&sv)[CHUNK][GPB]) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < CHUNK; ++c) {
            const int b = ks + (j + c) * KS;
            if (b >= KB) break;
            const char *x = lds + ((b - first) * 128 + 8 * q) * L::ES;
            const float *xs = xsums + (b - first) * GPB;
#pragma unroll
            for (int g = 0; g < GPB; ++g) {
                const float scale = __uint_as_float(sv[c][g] & ~15u), zero = (float)(sv[c][g] & 15u);
                float acc0;
                if constexpr (XT == DSQ_T_I8) {
                    v4i acc = {};
#pragma unroll
                    for (int t = g * SPG; t < (g + 1) * SPG; ++t)
                        acc = __builtin_amdgcn_mfma_i32_16x16x32_i8(*reinterpret_cast<const long *>(x + 32 * t), codes_i8(wv[c][t]), acc, 0, 0, 0);
                    acc0 = (float)acc[0];
                } else {
                    v4f acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int t = g * SPG; t < (g + 1) * SPG; ++t)
#pragma unroll
                        for (int p = L::TERMS - 1; p >= 0; --p) {
                            const char *f = x + p * plane + 64 * t;
                            if constexpr (XT == DSQ_T_F16)
                                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(*reinterpret_cast<const f16x8 *>(f), codes_f16(wv[c][t]), acc, 0, 0, 0);
                            else
                                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8 *>(f), codes_bf16(wv[c][t]), acc, 0, 0, 0);
                        }
                    acc0 = acc[0];
                }
                sum = __builtin_fmaf(scale, __builtin_fmaf(-zero, xs[g], acc0), sum);
            }
        }
    };
    // The row's blocks from `first` on to LDS, eight channels a thread and four loads under way, and their groups' sums.
    auto stage = [&](int first) __attribute__((always_inline)) {
        constexpr int AHEAD = 4;
        const int units = min(seg, KB - first) * 16;
        for (int u0 = threadIdx.x; u0 < units; u0 += 64 * WAVES * AHEAD) {
            Frag<XT> f[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int k = 128 * first + 8 * min(u0 + 64 * WAVES * i, units - 1);
                // (a row of codes ends with its pitch, and what lies behind K meets levels of 0)
                if (XT == DSQ_T_I8 || a.K >= 8) load_frag<XT, true>(f[i], a.x, XT == DSQ_T_I8 || k + 8 <= a.K ? k : 0, a.K, true);
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int u = u0 + 64 * WAVES * i, k = 128 * first + 8 * u;
                if (u >= units) break;
                if (XT != DSQ_T_I8 && k + 8 > a.K) load_frag<XT, false>(f[i], a.x, k, a.K, true);
                scale_up(f[i]);
                char *to = lds + 8 * u * L::ES;
                if constexpr (XT == DSQ_T_F32) {
                    bf16x8 t[3];
                    split3(f[i].v, t);
#pragma unroll
                    for (int p = 0; p < 3; ++p) *reinterpret_cast<bf16x8 *>(to + p * plane) = t[p];
                } else {
                    *reinterpret_cast<Frag<XT> *>(to) = f[i];
                }
                const float s = lanes_sum<4 * SPG>(sum8(f[i]));
                if (u % (4 * SPG) == 0) xsums[u / (4 * SPG)] = s;
            }
        }
    };

    v4u wa[CHUNK], wb[CHUNK];
    uint32_t sa[CHUNK][GPB], sb[CHUNK][GPB];
    const int per = seg / KS;                       // a wave's blocks of a segment
    int j = 0;
    load(0, wa, sa);
    load(CHUNK, wb, sb);
    for (int first = 0; first < KB; first += seg) {
        if (first > 0) __syncthreads();
        stage(first);
        __syncthreads();
        // (two sets of weight registers in turn; a segment holds an even number of chunks, or is the last)
        for (const int end = j + per; j < end && ks + j * KS < KB; j += 2 * CHUNK) {
            chunk(j, first, wa, sa);
            load(j + 2 * CHUNK, wa, sa);
            if (j + CHUNK < end) chunk(j + CHUNK, first, wb, sb);
            load(j + 3 * CHUNK, wb, sb);
        }
    }
    if (KS > 1) {
        __syncthreads();
        float *part = reinterpret_cast<float *>(lds);           // [wave][channel]
        if (lane < 16) part[wave * 16 + lane] = sum;
        __syncthreads();
        if (ks != 0) return;
        for (int p = 1; p < KS; ++p) sum += part[(wave + p) * 16 + r];
    }
    const int n = 16 * nt + r;
    if (mine >= tiles || n >= a.N || lane >= 16) return;
    if (XT == DSQ_T_F32) sum *= kDown;
    if constexpr (kSumsOverflow<XT>)
        if (__builtin_expect(overflowed(sum), 0)) sum = product_in_64_bits<XT>(0, n);
    if (XT == DSQ_T_I8) sum *= a.x_scale[0];
    if (a.bias) sum += load_out(a.bias, n, a.out_type);
    store_out(a.out, n, a.out_type, sum);
}

// A segment of the row that leaves room for a second workgroup on the compute unit.
constexpr int LDS_SHARED = 64 * 1024;

template <int XT, int GPB>
hipError_t launch_row(const DsqW4Args &a, hipStream_t stream)
{
    typedef Row<XT> L;
    const int KB = dsq_w4_round(a.K) / 128;
    const int64_t tiles = ((int64_t)a.N + 15) / 16;
    const int block = 128 * L::ES * L::TERMS + GPB * 4;
    // Two waves a SIMD keep the memory busy, and four where each still has 16 blocks (us, KS for 2048 / 4096 waves: 8192 -> 32768
    // 34.7 / 30.4, 4096 -> 12288 10.0 / 11.3)
    int KS = 1;
    while (KS < WAVES && (tiles * KS < 2048 || (tiles * KS < 4096 && KB / (2 * KS) >= 16))) KS *= 2;
    const int step = 2 * CHUNK * KS, all = (KB + step - 1) / step * step, most = LDS_SHARED / block / step * step;
    const int seg = all < most ? all : most;
    const dim3 grid((unsigned)((tiles + WAVES / KS - 1) / (WAVES / KS)));
    w4_row_kernel<XT, GPB><<<grid, 64 * WAVES, (size_t)seg * block, stream>>>(a, KS, seg);
    return hipGetLastError();
}

template <int XT>
hipError_t launch_groups(const DsqW4Args &a, hipStream_t stream)
{
    return a.group == 32 ? launch_row<XT, 4>(a, stream) : a.group == 64 ? launch_row<XT, 2>(a, stream) : launch_row<XT, 1>(a, stream);
}

}  // namespace

hipError_t dsq_launch_w4_row(const DsqW4Args &a, hipStream_t stream)
{
    switch (a.x_type) {
    case DSQ_T_F32: return launch_groups<DSQ_T_F32>(a, stream);
    case DSQ_T_F16: return launch_groups<DSQ_T_F16>(a, stream);
    case DSQ_T_BF16: return launch_groups<DSQ_T_BF16>(a, stream);
    }
    return launch_groups<DSQ_T_I8>(a, stream);
}
