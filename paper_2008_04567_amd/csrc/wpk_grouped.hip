// Products of rows sorted by expert in 32 and 16 bits: which of the kernels in wpk_product.h a call runs, and its checks.
#include "wpk_grouped.h"

namespace wpk {

template <typename T, bool GATED> static int grouped_typed(const LinearArgs &a, bool direct, hipStream_t st)
{
    const GroupedGrid g(a, 64, GATED ? 32 : 64);
    if (g.too_large(256)) return WPK_E_UNSUPPORTED;
    if constexpr (sizeof(T) == 2) {
        if (direct) {
            hipLaunchKernelGGL((grouped_direct_kernel<T, 64, 64, 2, 2, 64, 4, GATED>), dim3(g.all), dim3(256), 0, st, a);
            WPK_HIP(hipGetLastError());
            return WPK_OK;
        }
    }
    hipLaunchKernelGGL((grouped_tiles_kernel<T, 64, 64, 2, 2, GATED>), dim3(g.all), dim3(256), 0, st, a);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

static int check_grouped(const wpk_grouped_linear_desc *dp)
{
    if (!dp) return WPK_E_NULL_PTR;
    const wpk_grouped_linear_desc &d = *dp;
    const int64_t halves = d.gated ? 2 : 1, most = 1ll << 20, far = 1ll << 40;
    const bool q8 = d.dtype == WPK_E4M3;
    if (d.groups < 1 || d.rows < 0 || d.n < 1 || d.k < 1 || d.x_rows < 0 || d.x_stride < d.k || d.w_stride < d.k || d.y_stride < d.n)
        return WPK_E_BAD_DESC;
    if (d.groups > 4096 || d.rows > kMostRows || d.x_rows > kMostRows || d.n > kMostRows / 2 || (!q8 && !seq_type_ok(d.dtype)) ||
        !seq_type_ok(d.y_dtype) || (!q8 && d.y_dtype != d.dtype && d.y_dtype != WPK_F32) || d.act < WPK_ACT_NONE || d.act > WPK_ACT_GELU ||
        (d.gated != 0 && d.gated != 1) || d.reserved != 0 || d.x_stride >= most || d.w_stride >= most || d.y_stride >= most)
        return WPK_E_UNSUPPORTED;
    if (d.w_group_stride < halves * d.n * d.w_stride) return WPK_E_BAD_DESC;
    if (d.w_group_stride >= far) return WPK_E_UNSUPPORTED;
    if (q8) {
        if (d.x_scale_stride < scale_blocks(d.k) || d.w_scale_stride < scale_blocks(d.k)) return WPK_E_BAD_DESC;
        if (d.x_stride % 16 != 0 || d.w_stride % 16 != 0 || d.w_group_stride % 16 != 0 || d.x_scale_stride >= most || d.w_scale_stride >= most)
            return WPK_E_UNSUPPORTED;
        if (d.w_scale_group_stride < halves * scale_blocks(d.n) * d.w_scale_stride) return WPK_E_BAD_DESC;
        if (d.w_scale_group_stride >= far) return WPK_E_UNSUPPORTED;
    }
    return WPK_OK;
}

}  // namespace wpk

extern "C" {

int64_t wpk_grouped_linear_workspace_bytes(const wpk_grouped_linear_desc *d)
{
    return wpk::check_grouped(d);
}

int wpk_grouped_linear_fwd(const wpk_grouped_linear_desc *dp, const void *x, const float *x_scales, const void *w,
                           const float *w_scales, const int32_t *starts, const int32_t *source, void *y, void *workspace,
                           void *stream)
{
    using namespace wpk;
    const int rc = check_grouped(dp);
    if (rc != WPK_OK) return rc;
    const wpk_grouped_linear_desc d = *dp;
    if (d.rows == 0) return WPK_OK;
    if ((!starts && d.groups > 1) || d.x_rows < 1 || (!source && d.x_rows < d.rows)) return WPK_E_BAD_ARG;
    const bool q8 = d.dtype == WPK_E4M3;
    if (!x || !w || !y || (q8 && (!x_scales || !w_scales))) return WPK_E_NULL_PTR;
    const size_t e = q8 ? 16 : seq_type_bytes(d.dtype), ye = seq_type_bytes(d.y_dtype);
    if (!aligned_to(x, e) || !aligned_to(w, e) || !aligned_to(y, ye) || !aligned_to(starts, 4) || !aligned_to(source, 4) ||
        !aligned_to(x_scales, 4) || !aligned_to(w_scales, 4) || !aligned_to(workspace, 16) || (!q8 && (x_scales || w_scales)))
        return WPK_E_BAD_ARG;
    const bool wide = d.n % 4 == 0 && d.y_stride % 4 == 0 && aligned_to(y, 4 * ye);
    const LinearArgs a = {x, w, nullptr, nullptr, y, nullptr, d.rows, d.n, d.k, d.act, d.y_dtype == WPK_F32, 1, (d.k + 127) / 128 * 128,
                          64, wide, d.x_stride, d.w_stride, d.y_stride, d.y_stride, 0, starts, source, d.groups, d.x_rows,
                          d.w_group_stride};
    const hipStream_t st = (hipStream_t)stream;
    if (q8) {
        const Q8Args q = {a, x_scales, w_scales, d.x_scale_stride, d.w_scale_stride, d.w_scale_group_stride};
        return grouped_q8(q, d.y_dtype, d.gated != 0, st);
    }
    // Loads that write LDS move 16 aligned bytes, and reach 2^31 bytes from the first row where rows are looked up or a weight has
    // two halves.
    const int64_t x_bytes = (int64_t)d.x_rows * d.x_stride * (int64_t)e, w_bytes = 2 * (int64_t)d.n * d.w_stride * (int64_t)e;
    const bool direct = d.k % 8 == 0 && d.x_stride % 8 == 0 && d.w_stride % 8 == 0 && d.w_group_stride % 8 == 0 && aligned_to(x, 16) &&
                        aligned_to(w, 16) && (!source || x_bytes < 1ll << 31) && (!d.gated || w_bytes < 1ll << 31);
    if (d.dtype == WPK_BF16) return d.gated ? grouped_typed<bf16, true>(a, direct, st) : grouped_typed<bf16, false>(a, direct, st);
    if (d.dtype == WPK_F16) return d.gated ? grouped_typed<f16, true>(a, direct, st) : grouped_typed<f16, false>(a, direct, st);
    return d.gated ? grouped_typed<float, true>(a, false, st) : grouped_typed<float, false>(a, false, st);
}

}  // extern "C"
