// Matrix product y = act(x w^T + bias) + residual: which of the kernels in wpk_product.h a call runs, and its checks.
#include "wpk_product.h"

namespace wpk {

// ---- which of them ------------------------------------------------------------------------------------------------
// Rows of x that the row kernel takes.  32 rows by 8512 columns of 2048 take 10.8 us in bf16 and 26.5 in fp32, 65 (two rows of
// tiles) 15.4 and 50.  Between, neither way is the faster throughout; 64 rows by the row kernel and by tiles, us:
//   columns x reduction   1024 x 512   1024 x 2048   8512 x 512   8512 x 2048   4096 x 8192
//   bf16                   5.0   5.2   11.3    8.7    6.5   5.4   14.8   10.9   37.4   16.9
//   fp32                   7.8  16.8   24.2   19.9   22.7  16.8   48.2   32.8   81.2   45.6
// so tiles would gain where reductions are long, and lose half in fp32 where they are not.  (The row kernel's fp32 form for 33
// rows on keeps 6 to 62 registers in scratch memory.)
static const int kRowsMost = 64;
struct LinearShape {
    int tile;                         // rows and columns of a tile; 0: the row kernel
    int width;                        // of a workgroup of the row kernel
    int slices, slice_k;
};

static LinearShape linear_shape(const wpk_linear_desc &d)
{
    LinearShape s = {0, 0, 1, (d.k + 63) / 64 * 64};
    const int64_t steps = (d.k + 63) / 64;
    int64_t groups, slices;
    if (d.m <= kRowsMost) {
        // As many columns a workgroup as give every compute unit the same: 8512 columns of 2048 by 32 rows take 16.9 us in
        // workgroups of 32 (266 for 256 compute units) and 10.5 in such of 36.  At least as many as keep the reads of x, all
        // of which every workgroup does, small beside those of w.
        const int least = d.m <= 4 ? 4 : d.m <= 16 ? 8 : 16;
        const int64_t rounds = ((int64_t)d.n + 48 * kComputeUnits - 1) / (48 * kComputeUnits);
        const int64_t even = (d.n + rounds * kComputeUnits - 1) / (rounds * kComputeUnits);
        s.width = (int)((even > least ? even : least) + 3) / 4 * 4;
        groups = (d.n + s.width - 1) / s.width;
        // each of the eight waves keeps four runs of 64 at least
        slices = kComputeUnits / groups;
        if (slices > steps / (4 * kRowsWaves)) slices = steps / (4 * kRowsWaves);
    } else {
        auto tiles = [&](int t) { return (int64_t)((d.m + t - 1) / t) * ((d.n + t - 1) / t); };
        s.tile = d.dtype != WPK_F32 && tiles(256) >= kComputeUnits ? 256 : tiles(128) >= kComputeUnits / 2 ? 128 : 64;
        groups = tiles(s.tile);
        // fp32 wants several workgroups a compute unit, which cut their operands while others multiply
        slices = (d.dtype != WPK_F32 ? 1 : s.tile == 64 ? 3 : 2) * kComputeUnits / groups;
        if (slices > steps / 8) slices = steps / 8;
    }
    if (slices > 16) slices = 16;
    if (slices < 2) return s;
    s.slice_k = (int)((steps + slices - 1) / slices) * 64;
    s.slices = (d.k + s.slice_k - 1) / s.slice_k;
    return s;
}

static int64_t part_stride(const wpk_linear_desc &d) { return ((int64_t)d.n + 3) / 4 * 4; }

static int check_linear(const wpk_linear_desc *dp)
{
    if (!dp) return WPK_E_NULL_PTR;
    const wpk_linear_desc &d = *dp;
    if (d.m < 0 || d.n < 1 || d.k < 1 || d.x_stride < d.k || d.w_stride < d.k || d.y_stride < d.n || d.residual_stride < d.n)
        return WPK_E_BAD_DESC;
    const int64_t most = 1ll << 20;
    if (d.m > kMostRows || d.n > kMostRows || !seq_type_ok(d.dtype) || (d.y_dtype != d.dtype && d.y_dtype != WPK_F32) || d.act < WPK_ACT_NONE ||
        d.act > WPK_ACT_GELU || d.x_stride >= most || d.w_stride >= most || d.y_stride >= most || d.residual_stride >= most)
        return WPK_E_UNSUPPORTED;
    return WPK_OK;
}

template <typename T, int MT> static int launch_rows(const LinearArgs &a, hipStream_t st)
{
    const int kThreads = 64 * kRowsWaves, U = MT == 1 ? (sizeof(T) == 2 ? 4 : 2) : MT == 2 || sizeof(T) == 2 ? 2 : 1;
    const dim3 grid((a.n + a.width - 1) / a.width, a.slices);
    if (a.width <= 16) hipLaunchKernelGGL((linear_rows_kernel<T, MT, 1, U>), grid, dim3(kThreads), 0, st, a);
    else if (a.width <= 32) hipLaunchKernelGGL((linear_rows_kernel<T, MT, 2, U>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((linear_rows_kernel<T, MT, 3, U>), grid, dim3(kThreads), 0, st, a);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

template <typename T> static int launch_rows(const LinearArgs &a, hipStream_t st)
{
    return a.m <= 16 ? launch_rows<T, 1>(a, st) : a.m <= 32 ? launch_rows<T, 2>(a, st) : launch_rows<T, 4>(a, st);
}

static unsigned tile_count(const LinearArgs &a, int b) { return (unsigned)(((a.m + b - 1) / b) * ((a.n + b - 1) / b)); }

template <typename T> static int launch_tiles(const LinearArgs &a, int tile, bool direct, hipStream_t st)
{
    const dim3 grid(tile_count(a, tile), a.slices);
    if constexpr (sizeof(T) == 2) {
        if (direct) {
            if (tile == 256) hipLaunchKernelGGL((linear_direct_kernel<T, 256, 256, 2, 4, 64, 2>), grid, dim3(512), 0, st, a);
            // four steps' operands in LDS for a workgroup that has its compute unit to itself, two for two that share one
            else if (tile == 128 && grid.x * grid.y <= (unsigned)kComputeUnits)
                hipLaunchKernelGGL((linear_direct_kernel<T, 128, 128, 2, 4, 64, 4>), grid, dim3(512), 0, st, a);
            else if (tile == 128) hipLaunchKernelGGL((linear_direct_kernel<T, 128, 128, 2, 4, 64, 2>), grid, dim3(512), 0, st, a);
            else hipLaunchKernelGGL((linear_direct_kernel<T, 64, 64, 2, 2, 64, 4>), grid, dim3(256), 0, st, a);
            WPK_HIP(hipGetLastError());
            return WPK_OK;
        }
    }
    if (tile == 64) hipLaunchKernelGGL((linear_tiles_kernel<T, 64, 64, 2, 2>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((linear_tiles_kernel<T, 128, 128, 2, 2>), dim3(tile_count(a, 128), a.slices), dim3(256), 0, st, a);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

template <typename T> static int linear_typed(const LinearArgs &a, const LinearShape &s, bool direct, hipStream_t st)
{
    const int rc = s.tile == 0 ? launch_rows<T>(a, st) : launch_tiles<T>(a, s.tile, direct, st);
    if (rc != WPK_OK || a.slices == 1) return rc;
    const int64_t quads = (int64_t)((a.n + 3) / 4) * a.m;
    hipLaunchKernelGGL((linear_join_kernel<T>), dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, st, a);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

}  // namespace wpk

extern "C" {

int64_t wpk_linear_workspace_bytes(const wpk_linear_desc *d)
{
    const int rc = wpk::check_linear(d);
    if (rc != WPK_OK) return rc;
    const wpk::LinearShape s = wpk::linear_shape(*d);
    return s.slices < 2 ? 0 : (int64_t)s.slices * d->m * wpk::part_stride(*d) * (int64_t)sizeof(float);
}

int wpk_linear_fwd(const wpk_linear_desc *dp, const void *x, const void *w, const void *bias, const void *residual, void *y,
                   void *workspace, void *stream)
{
    using namespace wpk;
    const int rc = check_linear(dp);
    if (rc != WPK_OK) return rc;
    const wpk_linear_desc d = *dp;
    if (d.m == 0) return WPK_OK;
    if (!x || !w || !y) return WPK_E_NULL_PTR;
    const size_t e = seq_type_bytes(d.dtype), ye = seq_type_bytes(d.y_dtype);
    if (!aligned_to(x, e) || !aligned_to(w, e) || !aligned_to(bias, e) || !aligned_to(residual, e) || !aligned_to(y, ye))
        return WPK_E_BAD_ARG;
    const LinearShape s = linear_shape(d);
    if (s.slices > 1 && !workspace) return WPK_E_NULL_PTR;
    if (!aligned_to(workspace, 16)) return WPK_E_BAD_ARG;
    const bool wide = d.n % 4 == 0 && d.y_stride % 4 == 0 && aligned_to(y, 4 * ye) && aligned_to(bias, 4 * e) &&
                      (!residual || (d.residual_stride % 4 == 0 && aligned_to(residual, 4 * e)));
    LinearArgs a = {x, w, bias, residual, y, (float *)workspace, d.m, d.n, d.k, d.act, d.y_dtype == WPK_F32,
                    s.slices, s.slice_k, s.width, wide, d.x_stride, d.w_stride, d.y_stride, d.residual_stride, part_stride(d),
                    nullptr, nullptr, 1, d.m, 0};
    // (loads that write LDS move 16 aligned bytes)
    const bool direct = d.k % 8 == 0 && d.x_stride % 8 == 0 && d.w_stride % 8 == 0 && aligned_to(x, 16) && aligned_to(w, 16);
    const hipStream_t st = (hipStream_t)stream;
    if (d.dtype == WPK_BF16) return linear_typed<bf16>(a, s, direct, st);
    if (d.dtype == WPK_F16) return linear_typed<f16>(a, s, direct, st);
    return linear_typed<float>(a, s, direct, st);
}

}  // extern "C"
