// Matrix product y = act(x w^T + bias) + residual.
#include "wpk_seq.h"

namespace wpk {

struct LinearArgs {
    const void *x, *w, *bias, *residual;
    void *y;
    int32_t m, n, k, act, y_f32;
    int64_t x_stride, w_stride, y_stride, residual_stride;
};

// 64 x 64 outputs a workgroup, 4 x 4 a lane, operands through LDS 16 of the reduction at a time, fp32 multiply-adds.
template <typename T> __global__ void __launch_bounds__(256) linear_plain_kernel(LinearArgs a)
{
    __shared__ float xs[16][65], ws[16][65];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
    const T *x = (const T *)a.x, *w = (const T *)a.w;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < a.k; k0 += 16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = ty + 16 * i, kk = k0 + tx;
            xs[tx][row] = m0 + row < a.m && kk < a.k ? (float)x[(int64_t)(m0 + row) * a.x_stride + kk] : 0.0f;
            ws[tx][row] = n0 + row < a.n && kk < a.k ? (float)w[(int64_t)(n0 + row) * a.w_stride + kk] : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(xs[k][ty + 16 * i], ws[k][tx + 16 * j], acc[i][j]);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (m >= a.m || n >= a.n) continue;
            float v = acc[i][j];
            if (a.bias) v += (float)((const T *)a.bias)[n];
            v = a.y_f32 ? apply_act<float>(v, a.act) : apply_act<T>(v, a.act);
            if (a.residual) v += (float)((const T *)a.residual)[(int64_t)m * a.residual_stride + n];
            if (a.y_f32) ((float *)a.y)[(int64_t)m * a.y_stride + n] = v;
            else ((T *)a.y)[(int64_t)m * a.y_stride + n] = (T)v;
        }
}

static int check_linear(const wpk_linear_desc *dp)
{
    if (!dp) return WPK_E_NULL_PTR;
    const wpk_linear_desc &d = *dp;
    if (d.m < 0 || d.n < 1 || d.k < 1 || d.x_stride < d.k || d.w_stride < d.k || d.y_stride < d.n || d.residual_stride < d.n)
        return WPK_E_BAD_DESC;
    const int64_t most = 1ll << 20;
    if (!seq_type_ok(d.dtype) || (d.y_dtype != d.dtype && d.y_dtype != WPK_F32) || d.act < WPK_ACT_NONE ||
        d.act > WPK_ACT_GELU || d.x_stride >= most || d.w_stride >= most || d.y_stride >= most || d.residual_stride >= most)
        return WPK_E_UNSUPPORTED;
    return WPK_OK;
}

template <typename T> static int linear_typed(const LinearArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL((linear_plain_kernel<T>), dim3((a.n + 63) / 64, (a.m + 63) / 64), dim3(256), 0, st, a);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

}  // namespace wpk

extern "C" {

int64_t wpk_linear_workspace_bytes(const wpk_linear_desc *d)
{
    const int rc = wpk::check_linear(d);
    return rc == WPK_OK ? 0 : rc;
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
    const size_t e = seq_type_bytes(d.dtype);
    if (!aligned_to(x, e) || !aligned_to(w, e) || !aligned_to(bias, e) || !aligned_to(residual, e) ||
        !aligned_to(y, seq_type_bytes(d.y_dtype)))
        return WPK_E_BAD_ARG;
    LinearArgs a = {x, w, bias, residual, y, d.m, d.n, d.k, d.act, d.y_dtype == WPK_F32, d.x_stride, d.w_stride,
                    d.y_stride, d.residual_stride};
    const hipStream_t st = (hipStream_t)stream;
    if (d.dtype == WPK_BF16) return linear_typed<bf16>(a, st);
    if (d.dtype == WPK_F16) return linear_typed<f16>(a, st);
    return linear_typed<float>(a, st);
}

}  // extern "C"
