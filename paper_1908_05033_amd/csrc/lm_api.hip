// C ABI of the calls for language-model layers (see include/dsqconv.h): host-side validation and dispatch.
#include <math.h>

#include "../../include/dsqconv.h"
#include "dsq_kernels.h"
#include "lm_kernels.h"

namespace {

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }
bool type_ok(dsq_dtype t) { return t == DSQ_F32 || t == DSQ_F16 || t == DSQ_BF16; }
bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }
// The largest row length, output channel count and row count of these calls, and the most weights of a layer.
const int kMaxDim = 1 << 20, kMaxOut = 1 << 24, kMaxRows = 1 << 21;
bool weights_ok(int N, int K) { return N <= kMaxOut && K <= kMaxDim && (int64_t)dsq_w4_round(N) * dsq_w4_round(K) <= 1LL << 36; }

dsq_status of_hip(hipError_t e) { return e == hipSuccess ? DSQ_OK : DSQ_ERR_HIP; }

}  // namespace

extern "C" {

size_t dsq_code_row_bytes(int dim) { return dim <= 0 || dim > kMaxDim ? 0 : (size_t)dsq_w4_round(dim); }

size_t dsq_rms_norm_bwd_bytes(int rows, int dim)
{
    if (rows <= 0 || dim <= 0 || rows > kMaxRows || dim > kMaxDim) return 0;
    // (the types differ in the rows a workgroup takes: room for the most workgroups)
    int parts = 0;
    for (int t : {DSQ_T_F32, DSQ_T_F16, DSQ_T_BF16}) {
        const int p = dsq_rms_norm_bwd_parts(rows, dim, t);
        parts = p > parts ? p : parts;
    }
    return (size_t)parts * dim * 4;
}

size_t dsq_w4_packed_bytes(int N, int K)
{
    if (N <= 0 || K <= 0 || !weights_ok(N, K)) return 0;
    return (size_t)dsq_w4_round(N) * dsq_w4_round(K) / 2;
}

size_t dsq_w4_scale_bytes(int N, int K, int group)
{
    if (N <= 0 || K <= 0 || !weights_ok(N, K) || !group_ok(group)) return 0;
    return (size_t)dsq_w4_round(N) * (dsq_w4_round(K) / group) * 4;
}

dsq_status dsq_rms_norm(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride,
                        const void *weight, dsq_dtype dtype, int rows, int dim, float eps, void *sum, void *y,
                        int8_t *codes, size_t codes_bytes, float *scales, float *rstd, void *hip_stream)
{
    if (!type_ok(dtype)) return DSQ_ERR_UNSUPPORTED;
    if (rows < 0 || dim <= 0) return DSQ_ERR_SHAPE;
    if (rows > kMaxRows || dim > kMaxDim) return DSQ_ERR_UNSUPPORTED;
    if (!(eps > 0.0f && isfinite(eps))) return DSQ_ERR_RANGE;
    if (rows == 0) return DSQ_OK;
    if (!x || (codes && !scales) || (scales && !codes)) return DSQ_ERR_NULL;
    if (!sum && !y && !codes && !rstd) return DSQ_ERR_NULL;
    if (x_stride < 0 || (residual && residual_stride < 0)) return DSQ_ERR_SHAPE;
    if (!aligned16(x) || !aligned16(residual) || !aligned16(weight) || !aligned16(sum) || !aligned16(y) ||
        !aligned16(codes) || !aligned16(scales) || !aligned16(rstd))
        return DSQ_ERR_ALIGN;
    if (codes && codes_bytes < (size_t)rows * dsq_code_row_bytes(dim)) return DSQ_ERR_SIZE;
    // an output in the place of an input has to have its rows where the input has them
    if (rows > 1)
        for (void *o : {sum, y})
            if (o && ((o == x && x_stride != dim) || (o == residual && residual_stride != dim))) return DSQ_ERR_UNSUPPORTED;
    DsqNormArgs a;
    a.x = x; a.residual = residual; a.weight = weight;
    a.x_stride = x_stride; a.residual_stride = residual_stride;
    a.rows = rows; a.dim = dim; a.eps = eps;
    a.sum = sum; a.y = y; a.codes = codes; a.code_pitch = (int64_t)dsq_code_row_bytes(dim);
    a.scales = scales; a.rstd = rstd;
    return of_hip(dsq_launch_rms_norm(a, dtype, (hipStream_t)hip_stream));
}

dsq_status dsq_rms_norm_bwd(const void *h, int64_t h_stride, const void *weight, const float *rstd,
                            const void *grad_y, int64_t grad_y_stride, const void *grad_sum, int64_t grad_sum_stride,
                            dsq_dtype dtype, int rows, int dim, void *grad_x, float *grad_weight, void *workspace,
                            size_t workspace_bytes, void *hip_stream)
{
    if (!type_ok(dtype)) return DSQ_ERR_UNSUPPORTED;
    if (rows < 0 || dim <= 0) return DSQ_ERR_SHAPE;
    if (rows > kMaxRows || dim > kMaxDim) return DSQ_ERR_UNSUPPORTED;
    if (rows == 0) {
        if (!grad_weight) return DSQ_OK;
        if (!aligned16(grad_weight)) return DSQ_ERR_ALIGN;
        return of_hip(dsq_launch_fill_zero((int32_t *)grad_weight, (size_t)dim, (hipStream_t)hip_stream));
    }
    if (!h || !rstd || !grad_y || !grad_x || (grad_weight && !workspace)) return DSQ_ERR_NULL;
    if (h_stride < 0 || grad_y_stride < 0 || (grad_sum && grad_sum_stride < 0)) return DSQ_ERR_SHAPE;
    if (!aligned16(h) || !aligned16(weight) || !aligned16(rstd) || !aligned16(grad_y) || !aligned16(grad_sum) ||
        !aligned16(grad_x) || !aligned16(grad_weight) || !aligned16(workspace))
        return DSQ_ERR_ALIGN;
    if (grad_weight && workspace_bytes < dsq_rms_norm_bwd_bytes(rows, dim)) return DSQ_ERR_SIZE;
    if (rows > 1 && ((grad_x == h && h_stride != dim) || (grad_x == grad_y && grad_y_stride != dim) ||
                     (grad_x == grad_sum && grad_sum_stride != dim)))
        return DSQ_ERR_UNSUPPORTED;
    DsqNormBwdArgs a;
    a.h = h; a.weight = weight; a.rstd = rstd; a.grad_y = grad_y; a.grad_sum = grad_sum;
    a.h_stride = h_stride; a.grad_y_stride = grad_y_stride; a.grad_sum_stride = grad_sum_stride;
    a.rows = rows; a.dim = dim; a.grad_x = grad_x; a.grad_weight = grad_weight; a.partial = (float *)workspace;
    return of_hip(dsq_launch_rms_norm_bwd(a, dtype, (hipStream_t)hip_stream));
}

dsq_status dsq_pack_weights_w4(const float *w, const uint8_t *codes, const float *scale, const uint8_t *zero, int N, int K,
                               int group, void *w_packed, size_t w_bytes, void *w_scales, size_t scale_bytes,
                               void *hip_stream)
{
    if ((!w && !codes) || !w_packed || !w_scales) return DSQ_ERR_NULL;
    if ((codes && !scale) || (!scale != !zero)) return DSQ_ERR_NULL;
    if (w && codes) return DSQ_ERR_UNSUPPORTED;
    if (N <= 0 || K <= 0) return DSQ_ERR_SHAPE;
    if (!group_ok(group) || !weights_ok(N, K)) return DSQ_ERR_UNSUPPORTED;
    if (!aligned16(w) || !aligned16(codes) || !aligned16(scale) || !aligned16(zero) || !aligned16(w_packed) || !aligned16(w_scales))
        return DSQ_ERR_ALIGN;
    if (w_bytes < dsq_w4_packed_bytes(N, K) || scale_bytes < dsq_w4_scale_bytes(N, K, group)) return DSQ_ERR_SIZE;
    DsqW4PackArgs a;
    a.w = w; a.codes = codes; a.scale = scale; a.zero = zero;
    a.N = N; a.K = K; a.group = group; a.G = (K + group - 1) / group;
    a.packed = (uint32_t *)w_packed; a.scales = (uint32_t *)w_scales;
    return of_hip(dsq_launch_w4_pack(a, (hipStream_t)hip_stream));
}

}  // extern "C"

namespace {

dsq_status linear(DsqW4Args &a, dsq_dtype dtype, void *hip_stream)
{
    if (!type_ok(dtype)) return DSQ_ERR_UNSUPPORTED;
    if (a.M < 0 || a.N <= 0 || a.K <= 0) return DSQ_ERR_SHAPE;
    if (!group_ok(a.group) || a.M > kMaxRows || !weights_ok(a.N, a.K)) return DSQ_ERR_UNSUPPORTED;
    if (a.M == 0) return DSQ_OK;
    if (!a.x || !a.w || !a.scales || !a.out || (a.x_type == DSQ_T_I8 && !a.x_scale)) return DSQ_ERR_NULL;
    if (a.x_stride < 0 || (a.M > 1 && a.out_stride < a.N)) return DSQ_ERR_SHAPE;
    if (!aligned16(a.x) || !aligned16(a.x_scale) || !aligned16(a.w) || !aligned16(a.scales) || !aligned16(a.bias) || !aligned16(a.out))
        return DSQ_ERR_ALIGN;
    a.out_type = dtype;
    return of_hip(dsq_launch_w4_linear(a, (hipStream_t)hip_stream));
}

}  // namespace

extern "C" {

dsq_status dsq_linear_w4(const void *x, int64_t x_stride, dsq_dtype dtype, int M, int N, int K, int group,
                         const void *w_packed, const void *w_scales, const void *bias, void *out, int64_t out_stride,
                         void *hip_stream)
{
    DsqW4Args a;
    a.x = x; a.x_stride = x_stride; a.x_scale = nullptr; a.w = (const uint32_t *)w_packed; a.scales = (const uint32_t *)w_scales;
    a.bias = bias; a.out = out; a.out_stride = out_stride; a.M = M; a.N = N; a.K = K; a.group = group; a.x_type = dtype;
    return linear(a, dtype, hip_stream);
}

dsq_status dsq_linear_w4a8(const int8_t *codes, size_t codes_bytes, const float *code_scales, int M, int N, int K, int group,
                           const void *w_packed, const void *w_scales, const void *bias, dsq_dtype dtype, void *out,
                           int64_t out_stride, void *hip_stream)
{
    DsqW4Args a;
    a.x = codes; a.x_stride = (int64_t)dsq_code_row_bytes(K); a.x_scale = code_scales; a.w = (const uint32_t *)w_packed;
    a.scales = (const uint32_t *)w_scales; a.bias = bias; a.out = out; a.out_stride = out_stride;
    a.M = M; a.N = N; a.K = K; a.group = group; a.x_type = DSQ_T_I8;
    if (M > 0 && M <= kMaxRows && codes && codes_bytes < (size_t)M * dsq_code_row_bytes(K)) return DSQ_ERR_SIZE;
    return linear(a, dtype, hip_stream);
}

}  // extern "C"
