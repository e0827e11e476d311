// Packing of 4-bit weights with a scale and a zero point per group of input channels (once per layer).
//
// From floats, a group's range always holds 0: s = (max(w, 0) - min(w, 0)) / 15 in binary32, cut to 20 significant bits,
// z = rint(-min / s), code = clamp(rint(w / s) + z, 0, 15); a group of zeros has s = 0 and codes 0.  The level of a code is
// s * (code - z).
//
// A workgroup packs blocks of 16 output channels x 128 input channels, one after the other along the input channels: a thread
// takes eight input channels of one output channel, which are one word of the packed format (lm_kernels.h), so that rows are read
// 128 codes at a time and a block is written as 1 KB side by side; the threads of a group find its range by exchanges between
// lanes.  Bound by the way through memory: 32768 x 8192 codes 147 us (2.7 TB/s read and written), floats 264 us (4.6 TB/s).
#include "lm_device.h"

namespace {

constexpr int RUN = 8;       // blocks of a workgroup

__device__ __forceinline__ float cut_scale(float s)
{
    // the low four bits of the word hold the zero point: rounded to nearest, the step is at most 2^-20 of the scale off.  A lane
    // reads one word a group for both; what a group of 4-bit codes loses anyway, half a step, is 2^15 times as much.
    return __uint_as_float((__float_as_uint(s) + 8u) & ~15u);
}

template <int GROUP>
__global__ __launch_bounds__(256) void w4_pack_kernel(DsqW4PackArgs a)
{
    constexpr int LANES = GROUP / 8;                              // threads of a group, side by side
    const int KB = dsq_w4_round(a.K) / 128, Gp = KB * (128 / GROUP), runs = (KB + RUN - 1) / RUN;
    const int tile = (int)(blockIdx.x / runs), first = (int)(blockIdx.x % runs) * RUN, last = min(first + RUN, KB);
    const int r = threadIdx.x / 16, o = threadIdx.x % 16, n = 16 * tile + r;
    const size_t row = (size_t)n * a.K;
    for (int b = first; b < last; ++b) {
        const int k = 128 * b + 8 * o, g = k / GROUP;
        const int live = n < a.N ? min(max(a.K - k, 0), 8) : 0;   // channels of the thread that exist
        const bool grouped = n < a.N && g < a.G;
        float w[8] = {}, s = 0.0f;
        int z = 0;
        uint8_t c[8] = {};
        if (a.w) {
            if (live == 8) {
                const Side<float, 8> v = load_side<float, 8>(a.w + row + k);
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = v.at[i];
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < live) w[i] = a.w[row + k + i];
            }
        } else {
            if (live == 8) {
                const Side<uint8_t, 8> v = load_side<uint8_t, 8>(a.codes + row + k);
#pragma unroll
                for (int i = 0; i < 8; ++i) c[i] = v.at[i];
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < live) c[i] = a.codes[row + k + i];
            }
        }
        if (a.scale) {
            if (grouped) {
                s = cut_scale(a.scale[(size_t)n * a.G + g]);
                z = min((int)a.zero[(size_t)n * a.G + g], 15);
            }
        } else {
            // (channels that do not exist are 0 here, which the range holds anyway)
            float lo = 0.0f, hi = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                lo = fminf(lo, w[i]);
                hi = fmaxf(hi, w[i]);
            }
#pragma unroll
            for (int by = 1; by < LANES; by *= 2) {
                lo = fminf(lo, __shfl_xor(lo, by));
                hi = fmaxf(hi, __shfl_xor(hi, by));
            }
            s = cut_scale((hi - lo) / 15.0f);
            z = s > 0.0f ? (int)fminf(fmaxf(rintf(-lo / s), 0.0f), 15.0f) : 0;
        }
        if (o % LANES == 0) a.scales[((size_t)tile * Gp + g) * 16 + r] = __float_as_uint(s) | (uint32_t)z;
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int code = z;                                         // behind the last channel: level 0
            if (i < live) {
                if (!a.w) code = min((int)c[i], 15);
                else if (s != 0.0f) code = (int)fminf(fmaxf(rintf(w[i] / s) + (float)z, 0.0f), 15.0f);
            }
            word |= (uint32_t)code << (8 * (i & 3) + 4 * (i >> 2));
        }
        a.packed[(((size_t)tile * KB + b) * 64 + 16 * (o % 4) + r) * 4 + o / 4] = word;
    }
}

}  // namespace

hipError_t dsq_launch_w4_pack(const DsqW4PackArgs &a, hipStream_t stream)
{
    const int64_t runs = (dsq_w4_round(a.K) / 128 + RUN - 1) / RUN;
    const unsigned grid = (unsigned)(dsq_w4_round(a.N) / 16 * runs);
    if (a.group == 32) w4_pack_kernel<32><<<grid, 256, 0, stream>>>(a);
    else if (a.group == 64) w4_pack_kernel<64><<<grid, 256, 0, stream>>>(a);
    else w4_pack_kernel<128><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}
