// Products of rows sorted by expert in 32 and 16 bits: which of the kernels in wpk_product.h a call runs, and its checks.
#include "wpk_grouped.h"

namespace wpk {

template <typename T, bool GATED> static int launch_grouped_rows(LinearArgs a, hipStream_t st)
{
    const int U = sizeof(T) == 2 ? 4 : 2;
    a.width = GATED ? 16 : 32;
    const GroupedGrid g(a, 16, a.width);
    if (g.tiles * 64 * kRowsWaves >= 1ll << 32) return WPK_E_UNSUPPORTED;
    hipLaunchKernelGGL((grouped_rows_kernel<T, 1, 2, U, GATED>), dim3((unsigned)g.tiles), dim3(64 * kRowsWaves), 0, st, a);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

template <typename T, int B, int WM, int WN, int STAGES, bool GATED> static int launch_grouped_direct(const LinearArgs &a, hipStream_t st)
{
    const GroupedGrid g(a, B, GATED ? B / 2 : B);
    if (g.tiles * 64 * WM * WN >= 1ll << 32) return WPK_E_UNSUPPORTED;
    hipLaunchKernelGGL((grouped_direct_kernel<T, B, B, WM, WN, 64, STAGES, GATED>), dim3((unsigned)g.tiles), dim3(64 * WM * WN), 0, st, a);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

template <typename T, int B, bool GATED> static int launch_grouped_tiles(const LinearArgs &a, hipStream_t st)
{
    const GroupedGrid g(a, B, GATED ? B / 2 : B);
    if (g.tiles * 256 >= 1ll << 32) return WPK_E_UNSUPPORTED;
    hipLaunchKernelGGL((grouped_tiles_kernel<T, B, B, 2, 2, GATED>), dim3((unsigned)g.tiles), dim3(256), 0, st, a);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

// By the mean of the experts' rows and the workgroups there would be.  us, experts x columns x reduction (gated: twice the columns),
// rows of uneven spread:
//   bf16, rows kernel / tiles of 64 / 128 (two steps in LDS) / 256
//     8 x 2048 x 2048           mean 1: 13 / 13 / 24 / 39      64: 58 / 23 / 36 / 55     256: - / 55 / 47 / 64    1024: - / 176 / 117 / 120
//     64 x 1024 x 2048, gated   mean 4: 95 / 105 / 121 / 134   64: 439 / 144 / 154 / 184  128: 826 / 209 / 169 / 193   256: - / 354 / 241 / 213
//     64 x 2048 x 1536          mean 4: 82 / 75               64 x 2048 x 1024           mean 4: 58 / 55
//     16 x 4096 x 4096          mean 1: 59 / 76               4: 90 / 100
//     7 x 300 x 520             mean 95: 6.5 / 6.9 / 10
//   (mean <= 4 with k >= 2048 stands on the means of 1 and 4; where between 4 and 64 the two cross at such sizes was not measured)
//   (128 with four steps in LDS, for workgroups that have a compute unit to themselves: 8 x 2048 x 2048, mean 128, 26 against 37)
//   fp32, rows kernel / tiles of 64 / 128
//     8 x 2048 x 2048           mean 1: 28 / 74 / 115          32: 77 / 77 / 118         64: 116 / 79 / 119
//     64 x 1024 x 2048, gated   mean 8: 215 / 232 / 301        16: 295 / 256 / 299       128: 1630 / 654 / 530
//     128 x 768 x 1024, gated   mean 4: 169 / 168 / 228        8: 202 / 180 / 234        16: 274 / 193 / 235
//     16 x 2008 x 1024          mean 13: 46 / 47              20: 55 / 48               30: 73 / 49
//     32 x 512 x 512            mean 16: 16 / 18 / 37         64: 33 / 23 / 39
//     7 x 300 x 520             mean 95: 10 / 19 / 41
template <typename T, bool GATED> static int grouped_typed(const LinearArgs &a, bool direct, hipStream_t st)
{
    const int64_t rows = a.m, groups = a.groups, mean = rows / groups, out = GATED ? 16 : 32;
    const int64_t few = ((groups < rows ? groups : rows) + rows / 16) * ((a.n + out - 1) / out);     // workgroups of the row kernel
    auto columns = [&](int64_t b) { return GATED ? (a.n + b / 2 - 1) / (b / 2) : (a.n + b - 1) / b; };
    if constexpr (sizeof(T) == 2) {
        if (direct) {
            if (few <= 2 * kComputeUnits || (mean <= 4 && a.k >= 2048)) return launch_grouped_rows<T, GATED>(a, st);
            if (mean >= 256 && rows / 256 * columns(256) >= kComputeUnits) return launch_grouped_direct<T, 256, 2, 4, 2, GATED>(a, st);
            if (mean >= 96 && GroupedGrid(a, 128, GATED ? 64 : 128).tiles <= kComputeUnits)
                return launch_grouped_direct<T, 128, 2, 4, 4, GATED>(a, st);
            if (mean >= 96) return launch_grouped_direct<T, 128, 2, 4, 2, GATED>(a, st);
            return launch_grouped_direct<T, 64, 2, 2, 4, GATED>(a, st);
        }
    }
    if (mean <= 8 || few <= 8 * kComputeUnits) return launch_grouped_rows<T, GATED>(a, st);
    if (mean >= 128 && rows / 128 * columns(128) >= 2 * kComputeUnits) return launch_grouped_tiles<T, 128, GATED>(a, st);
    return launch_grouped_tiles<T, 64, GATED>(a, st);
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
