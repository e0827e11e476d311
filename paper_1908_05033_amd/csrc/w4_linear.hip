// Rows times group-scaled 4-bit weights:  out[m][n] = sum over groups g of s[n][g] * sum over k in g of (code - z) x[m][k].
// The kernel for few rows, and the choice of the kernel.
//
// The sum of a group runs on the 16x16x32 matrix instructions with exact operands: a code is converted to the type of
// x (a byte 0..15 is the e4m3 number code * 2^-9, which one instruction turns into bf16 or f16 times 2^9), binary32
// activations are cut into three bf16 terms, 8-bit rows meet the codes as bytes.  A matrix product with ones gives the
// group's sum of x for the zero points.  Groups are joined in binary32.
//
// A workgroup owns 16 output channels and 16 * MT rows; its waves share out the blocks of 128 input channels and join
// their sums in LDS, in a fixed order.
#include "w4_device.h"

namespace {

constexpr int ROWS_WAVES = 8;

// GPB: groups in a block of 128 channels.
template <int XT, int MT, int GPB>
__global__ __launch_bounds__(64 * ROWS_WAVES) void w4_rows_kernel(DsqW4Args a)
{
    constexpr int SPG = 4 / GPB;                    // steps of a group
    constexpr int CHUNK = MT == 1 ? 4 : 2;          // blocks whose weights are in flight together
    __shared__ v4f part[ROWS_WAVES][MT][64];
    const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int nt = blockIdx.x;
    const int64_t m0 = (int64_t)blockIdx.y * 16 * MT;
    const int KB = dsq_w4_round(a.K) / 128, Gp = KB * GPB;
    const v4u *w = reinterpret_cast<const v4u *>(a.w) + (size_t)nt * KB * 64 + lane;
    const uint32_t *sc = a.scales + (size_t)nt * Gp * 16 + r;
    const size_t e = XT == DSQ_T_F32 ? 4 : XT == DSQ_T_I8 ? 1 : 2;
    v4f sum[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) sum[i] = (v4f){0.f, 0.f, 0.f, 0.f};
    for (int b0 = wave; b0 < KB; b0 += ROWS_WAVES * CHUNK) {
        v4u wv[CHUNK];
        uint32_t sv[CHUNK][GPB];
#pragma unroll
        for (int j = 0; j < CHUNK; ++j) {
            const int b = min(b0 + j * ROWS_WAVES, KB - 1);       // (past the end: loaded and not used)
            wv[j] = w[(size_t)b * 64];
#pragma unroll
            for (int g = 0; g < GPB; ++g) sv[j][g] = sc[(size_t)(b * GPB + g) * 16];
        }
#pragma unroll
        for (int j = 0; j < CHUNK; ++j) {
            const int b = b0 + j * ROWS_WAVES;
            if (b >= KB) break;
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int64_t m = m0 + 16 * i + r;
                const void *row = (const char *)a.x + m * a.x_stride * (int64_t)e;
                Frag<XT> f[4];
                if (128 * (b + 1) <= a.K)
#pragma unroll
                    for (int t = 0; t < 4; ++t) f[t] = load_frag<XT, true>(row, 128 * b + 32 * t + 8 * q, a.K, m < a.M);
                else
#pragma unroll
                    for (int t = 0; t < 4; ++t) f[t] = load_frag<XT, false>(row, 128 * b + 32 * t + 8 * q, a.K, m < a.M);
#pragma unroll
                for (int g = 0; g < GPB; ++g) {
                    Sums<XT> s = {};
#pragma unroll
                    for (int t = 0; t < SPG; ++t) step<XT>(wv[j][g * SPG + t], f[g * SPG + t], s);
                    const float scale = __uint_as_float(sv[j][g] & ~15u), zero = (float)(sv[j][g] & 15u);
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        sum[i][c] = __builtin_fmaf(scale, __builtin_fmaf(-zero, (float)s.xs[c], (float)s.acc[c]), sum[i][c]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) part[wave][i][lane] = sum[i];
    __syncthreads();
    const int n = 16 * nt + r;
    for (int i = wave; i < MT; i += ROWS_WAVES) {
        v4f v = part[0][i][lane];
#pragma unroll
        for (int p = 1; p < ROWS_WAVES; ++p) v += part[p][i][lane];
        if (n >= a.N) continue;
        const float bias = a.bias ? load_out(a.bias, n, a.out_type) : 0.0f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int64_t m = m0 + 16 * i + 4 * q + c;
            if (m >= a.M) continue;
            float o = XT == DSQ_T_I8 ? v[c] * a.x_scale[m] : v[c];
            if (a.bias) o += bias;
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
    if (a.M > 64 && a.x_type != DSQ_T_F32) return dsq_launch_w4_tiles(a, stream);
    switch (a.x_type) {
    case DSQ_T_F32: return launch_of<DSQ_T_F32>(a, stream);
    case DSQ_T_F16: return launch_of<DSQ_T_F16>(a, stream);
    case DSQ_T_BF16: return launch_of<DSQ_T_BF16>(a, stream);
    }
    return launch_of<DSQ_T_I8>(a, stream);
}
