// Selective state space scan: a state of head_dim x state_dim numbers per head, forgotten by exp(delta a) and fed by
// delta x (outer) B at every token, read out by C.
#include "wpk_seq.h"

namespace wpk {

static const int kMaxHeadDim = 256, kMaxStateDim = 256;

template <typename T> struct SsmArgs {
    const T *x, *dt, *b, *c, *z;
    const float *a, *d_skip, *dt_bias, *state_in;
    float *state_out;
    T *y;
    Requests rq;
    int32_t heads, head_dim, groups, state_dim, softplus;
    int64_t x_stride, dt_stride, b_stride, c_stride, z_stride, y_stride;
};

// One wave per row of a head's state (head_dim rows of state_dim numbers, up to four a lane), token by token.
template <typename T> __global__ void __launch_bounds__(256) ssm_rows_kernel(SsmArgs<T> a)
{
    const int lane = threadIdx.x & 63, p = blockIdx.x * 4 + (threadIdx.x >> 6), head = blockIdx.y, r = blockIdx.z;
    if (p >= a.head_dim) return;
    int first, length;
    request_rows(a.rq, r, &first, &length);
    const int slot = request_slot(a.rq, r);
    const bool resume = a.state_in && slot >= 0 && (!a.rq.resume || a.rq.resume[r] != 0);
    const size_t at = (((size_t)max(slot, 0) * a.heads + head) * a.head_dim + p) * a.state_dim;
    const int N = a.state_dim, group = head / (a.heads / a.groups);
    float h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = resume && lane + 64 * i < N ? a.state_in[at + lane + 64 * i] : 0.0f;
    const float decay_rate = a.a[head], skip = a.d_skip ? a.d_skip[head] : 0.0f;
    const float bias = a.dt_bias ? a.dt_bias[head] : 0.0f;
    for (int t = first; t < first + length; ++t) {
        float delta = (float)a.dt[(int64_t)t * a.dt_stride + head] + bias;
        if (a.softplus) delta = softplus(delta);
        const float keep = expf(delta * decay_rate);
        const float x = (float)a.x[(int64_t)t * a.x_stride + (int64_t)head * a.head_dim + p];
        const float in = delta * x;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = lane + 64 * i;
            if (n < N) {
                h[i] = keep * h[i] + in * (float)a.b[(int64_t)t * a.b_stride + group * N + n];
                s = fmaf(h[i], (float)a.c[(int64_t)t * a.c_stride + group * N + n], s);
            }
        }
#pragma unroll
        for (int m = 32; m > 0; m >>= 1) s += __shfl_xor(s, m);
        if (lane == 0) {
            if (a.d_skip) s += skip * x;
            if (a.z) s *= silu_as<T>((float)a.z[(int64_t)t * a.z_stride + (int64_t)head * a.head_dim + p]);
            a.y[(int64_t)t * a.y_stride + (int64_t)head * a.head_dim + p] = (T)s;
        }
    }
    if (a.state_out && slot >= 0)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 64 * i < N) a.state_out[at + lane + 64 * i] = h[i];
}

static int check_ssm(const wpk_ssm_desc *dp)
{
    if (!dp) return WPK_E_NULL_PTR;
    const wpk_ssm_desc &d = *dp;
    if (d.sequences < 0 || d.tokens < 0 || d.max_length < 1 || d.heads < 1 || d.head_dim < 1 || d.groups < 1 ||
        d.state_dim < 1 || d.slots < 0 || d.heads % d.groups != 0)
        return WPK_E_BAD_DESC;
    const int64_t hp = (int64_t)d.heads * d.head_dim, gn = (int64_t)d.groups * d.state_dim;
    if (d.x_stride < hp || d.z_stride < hp || d.y_stride < hp || d.b_stride < gn || d.c_stride < gn || d.dt_stride < d.heads)
        return WPK_E_BAD_DESC;
    const int64_t most = 1ll << 22;
    if (!seq_type_ok(d.dtype) || d.dt_softplus < 0 || d.dt_softplus > 1 || d.head_dim > kMaxHeadDim ||
        d.state_dim > kMaxStateDim || d.sequences > 65535 || d.heads > 65535 || d.x_stride >= most || d.dt_stride >= most ||
        d.b_stride >= most || d.c_stride >= most || d.z_stride >= most || d.y_stride >= most)
        return WPK_E_UNSUPPORTED;
    return WPK_OK;
}

template <typename T>
static int ssm_typed(const wpk_ssm_desc &d, const void *x, const void *dt, const float *a, const void *b, const void *c,
                     const float *d_skip, const void *z, const float *dt_bias, const Requests &rq, const float *state_in,
                     float *state_out, void *y, hipStream_t st)
{
    SsmArgs<T> args = {(const T *)x, (const T *)dt, (const T *)b, (const T *)c, (const T *)z, a, d_skip, dt_bias, state_in,
                       state_out, (T *)y, rq, d.heads, d.head_dim, d.groups, d.state_dim, d.dt_softplus,
                       d.x_stride, d.dt_stride, d.b_stride, d.c_stride, d.z_stride, d.y_stride};
    hipLaunchKernelGGL((ssm_rows_kernel<T>), dim3((d.head_dim + 3) / 4, d.heads, d.sequences), dim3(256), 0, st, args);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

static int ssm_call(const wpk_ssm_desc *dp, bool step, const void *x, const void *dt, const float *a, const void *b,
                    const void *c, const float *d_skip, const void *z, const float *dt_bias, const int32_t *starts,
                    const int32_t *slot_map, const int32_t *resume, const float *state_in, float *state_out, void *y,
                    void *workspace, void *stream)
{
    int rc = check_ssm(dp);
    if (rc != WPK_OK) return rc;
    const wpk_ssm_desc d = *dp;
    rc = check_requests(d.sequences, d.tokens, d.max_length, d.slots, step, starts, slot_map, resume, state_in, state_out, 4);
    if (rc != WPK_OK) return rc;
    if (d.sequences == 0) return WPK_OK;
    if (!a || (d.tokens > 0 && (!x || !dt || !b || !c || !y))) return WPK_E_NULL_PTR;
    const size_t e = seq_type_bytes(d.dtype);
    if (!aligned_to(x, e) || !aligned_to(dt, e) || !aligned_to(b, e) || !aligned_to(c, e) || !aligned_to(z, e) ||
        !aligned_to(y, e) || !aligned_to(a, 4) || !aligned_to(d_skip, 4) || !aligned_to(dt_bias, 4))
        return WPK_E_BAD_ARG;
    const Requests rq = {starts, slot_map, resume, d.tokens, d.max_length, d.slots};
    const hipStream_t st = (hipStream_t)stream;
    if (d.dtype == WPK_BF16) return ssm_typed<bf16>(d, x, dt, a, b, c, d_skip, z, dt_bias, rq, state_in, state_out, y, st);
    if (d.dtype == WPK_F16) return ssm_typed<f16>(d, x, dt, a, b, c, d_skip, z, dt_bias, rq, state_in, state_out, y, st);
    return ssm_typed<float>(d, x, dt, a, b, c, d_skip, z, dt_bias, rq, state_in, state_out, y, st);
}

}  // namespace wpk

extern "C" {

int64_t wpk_ssm_workspace_bytes(const wpk_ssm_desc *d)
{
    const int rc = wpk::check_ssm(d);
    return rc == WPK_OK ? 0 : rc;
}

int wpk_ssm_scan_fwd(const wpk_ssm_desc *d, const void *x, const void *dt, const float *a, const void *b, const void *c,
                     const float *d_skip, const void *z, const float *dt_bias, const int32_t *starts, const int32_t *slot_map,
                     const int32_t *resume, const float *state_in, float *state_out, void *y, void *workspace, void *stream)
{
    return wpk::ssm_call(d, false, x, dt, a, b, c, d_skip, z, dt_bias, starts, slot_map, resume, state_in, state_out, y,
                         workspace, stream);
}

int wpk_ssm_scan_step(const wpk_ssm_desc *d, const void *x, const void *dt, const float *a, const void *b, const void *c,
                      const float *d_skip, const void *z, const float *dt_bias, const int32_t *slot_map,
                      const float *state_in, float *state_out, void *y, void *stream)
{
    return wpk::ssm_call(d, true, x, dt, a, b, c, d_skip, z, dt_bias, nullptr, slot_map, nullptr, state_in, state_out, y,
                         nullptr, stream);
}

}  // extern "C"
