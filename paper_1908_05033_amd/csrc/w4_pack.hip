// Packing of 4-bit weights with a scale and a zero point per group of input channels (cold: once per layer).
//
// From floats, a group's range always holds 0: s = (max(w, 0) - min(w, 0)) / 15 in binary32, cut to 20 significant bits,
// z = rint(-min / s), code = clamp(rint(w / s) + z, 0, 15); a group of zeros has s = 0 and codes 0.  The level of a code is
// s * (code - z).  One thread per channel and group: its codes are whole words of the packed format (lm_kernels.h).
#include "lm_device.h"

namespace {

__device__ __forceinline__ float cut_scale(float s)
{
    // the low four bits of the word hold the zero point: rounded to nearest, the step is at most 2^-20 of the scale off
    return __uint_as_float((__float_as_uint(s) + 8u) & ~15u);
}

template <int GROUP>
__global__ __launch_bounds__(256) void w4_pack_kernel(DsqW4PackArgs a)
{
    const int Gp = dsq_w4_round(a.K) / GROUP, KB = dsq_w4_round(a.K) / 128, Np = dsq_w4_round(a.N);
    const size_t id = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= (size_t)Np * Gp) return;
    const int n = (int)(id / Gp), g = (int)(id % Gp);
    const int k0 = g * GROUP, k1 = min(k0 + GROUP, a.K);
    const bool live = n < a.N && k0 < a.K;
    float s = 0.0f;
    int z = 0;
    if (live) {
        if (a.scale) {
            s = cut_scale(a.scale[(size_t)n * a.G + g]);
            z = min((int)a.zero[(size_t)n * a.G + g], 15);
        } else {
            float lo = 0.0f, hi = 0.0f;
            for (int k = k0; k < k1; ++k) {
                const float v = a.w[(size_t)n * a.K + k];
                lo = fminf(lo, v);
                hi = fmaxf(hi, v);
            }
            s = cut_scale((hi - lo) / 15.0f);
            z = s > 0.0f ? (int)fminf(fmaxf(rintf(-lo / s), 0.0f), 15.0f) : 0;
        }
    }
    a.scales[((size_t)(n / 16) * Gp + g) * 16 + n % 16] = __float_as_uint(s) | (uint32_t)z;
    for (int o = 0; o < GROUP / 8; ++o) {
        uint32_t word = 0;
        for (int i = 0; i < 8; ++i) {
            const int k = k0 + 8 * o + i;
            int c = z;                       // behind the last channel: level 0
            if (live && k < k1) {
                if (a.codes) c = min((int)a.codes[(size_t)n * a.K + k], 15);
                else if (s != 0.0f) c = (int)fminf(fmaxf(rintf(a.w[(size_t)n * a.K + k] / s) + (float)z, 0.0f), 15.0f);
                else c = z;
            }
            word |= (uint32_t)c << (8 * (i & 3) + 4 * (i >> 2));
        }
        const int k = k0 + 8 * o, lane = 16 * (k / 8 % 4) + n % 16;
        a.packed[(((size_t)(n / 16) * KB + k / 128) * 64 + lane) * 4 + k % 128 / 32] = word;
    }
}

}  // namespace

hipError_t dsq_launch_w4_pack(const DsqW4PackArgs &a, hipStream_t stream)
{
    const size_t threads = (size_t)dsq_w4_round(a.N) * (dsq_w4_round(a.K) / a.group);
    const unsigned grid = (unsigned)((threads + 255) / 256);
    if (a.group == 32) w4_pack_kernel<32><<<grid, 256, 0, stream>>>(a);
    else if (a.group == 64) w4_pack_kernel<64><<<grid, 256, 0, stream>>>(a);
    else w4_pack_kernel<128><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}
