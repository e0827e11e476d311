// Internal launch interface of the calls for language-model layers (lm_api.hip): RMS norm and products with
// group-scaled 4-bit weights.  Arguments have already been validated by the caller.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

// Element types in the order of dsq_dtype, and 8-bit codes.
enum { DSQ_T_F32 = 0, DSQ_T_F16 = 1, DSQ_T_BF16 = 2, DSQ_T_I8 = 3 };

struct DsqNormArgs {
    const void *x, *residual, *weight;       // residual and weight may be null
    int64_t x_stride, residual_stride;       // elements from row to row
    int rows, dim;
    float eps;
    void *sum, *y;                           // may be null
    int8_t *codes;                           // [rows][code_pitch] or null
    int64_t code_pitch;                      // bytes, a multiple of 128
    float *scales, *rstd;                    // may be null
};
hipError_t dsq_launch_rms_norm(const DsqNormArgs &a, int type, hipStream_t stream);

struct DsqNormBwdArgs {
    const void *h, *weight;                  // weight may be null
    const float *rstd;
    const void *grad_y, *grad_sum;           // grad_sum may be null
    int64_t h_stride, grad_y_stride, grad_sum_stride;
    int rows, dim;
    void *grad_x;
    float *grad_weight;                      // may be null
    float *partial;                          // [dsq_rms_norm_bwd_parts][dim], unused without grad_weight
};
// Workgroups of the backward pass, each of which leaves one row of partial sums.
int dsq_rms_norm_bwd_parts(int rows, int dim, int type);
hipError_t dsq_launch_rms_norm_bwd(const DsqNormBwdArgs &a, int type, hipStream_t stream);

// ---- 4-bit weights with a scale and a zero point per group of input channels ----------------------
//
// Codes: blocks of 16 output channels x 128 input channels, [Np/16][Kp/128][64 lanes][4 words], Np and Kp rounded
// up to 128; word t of lane 16q + r holds input channels 32t + 8q + 0..7 of output channel r, byte j = c[j] | c[j+4] << 4:
// the order in which lanes of the 16x16x32 matrix instructions take a step of 32 channels.
// Scales: [Np/16][Kp/group][16] words, a binary32 number whose low four bits are the zero point.
__host__ __device__ constexpr int dsq_w4_round(int n) { return (n + 127) / 128 * 128; }

struct DsqW4PackArgs {
    const float *w;                          // [N][K], or null with codes
    const uint8_t *codes;                    // [N][K], or null
    const float *scale;                      // [N][G]; null: from w
    const uint8_t *zero;                     // [N][G]; null: from w
    int N, K, group, G;
    uint32_t *packed, *scales;
};
hipError_t dsq_launch_w4_pack(const DsqW4PackArgs &a, hipStream_t stream);

struct DsqW4Args {
    const void *x;                           // [M] rows of x_stride elements
    int64_t x_stride;
    const float *x_scale;                    // 8-bit rows: one a row
    const uint32_t *w, *scales;
    const void *bias;                        // of out_type, or null
    void *out;
    int64_t out_stride;
    int M, N, K, group;
    int x_type, out_type;
};
hipError_t dsq_launch_w4_linear(const DsqW4Args &a, hipStream_t stream);
// The kernels for one row and for a few rows; those for many stand beside the choice.
hipError_t dsq_launch_w4_row(const DsqW4Args &a, hipStream_t stream);
hipError_t dsq_launch_w4_rows(const DsqW4Args &a, hipStream_t stream);
