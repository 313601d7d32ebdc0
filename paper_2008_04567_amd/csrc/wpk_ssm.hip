// Selective state space scan: a state of head_dim x state_dim numbers per head, forgotten by exp(delta a) and fed by
// delta x (outer) B at every token, read out by C.
#include "wpk_ssm_scan.h"

namespace wpk {

static const int kMaxHeadDim = 256, kMaxStateDim = 256;

// ---- single tokens -----------------------------------------------------------------------------------------
// Bound by the states, read and written once: 8 bytes a state element against 5 operations.  A workgroup takes U rows a
// lane group of one head: LPR lanes hold a row of state_dim numbers, V = 4 (16 bytes) or 1 a lane and CI times that, so
// every lane has U loads in flight before it needs the first.  Everything goes through buffer descriptors, an absent tensor
// being one of no bytes: a branch around loads makes the compiler wait for what is under way at its end.  The states are
// streamed (non-temporal): they are not wanted again before the next token.  256 requests of 64 heads of 64 x 128 numbers:
// 193 us, 5.6 TB/s, which is what a large copy reaches.
static const int kStream = 2;         // the buffer instructions' non-temporal bit

template <typename T, int V, int CI, int U> __global__ void __launch_bounds__(256, 4) ssm_step_kernel(SsmArgs<T> a, int lpr_log)
{
    typedef float vec __attribute__((ext_vector_type(V)));
    const int head = blockIdx.x, r = blockIdx.y, N = a.state_dim, P = a.head_dim;
    const int lpr = 1 << lpr_log, rows = 256 >> lpr_log;            // rows that a pass of the workgroup holds
    const int at_n = (threadIdx.x & (lpr - 1)) * V;
    const int p0 = blockIdx.z * U * rows + (threadIdx.x >> lpr_log);
    int first, length;
    request_rows(a.rq, r, &first, &length);
    const int slot = request_slot(a.rq, r);
    const size_t at = ((size_t)max(slot, 0) * a.heads + head) * P * N;
    const Rows in = rows_at(a.state_in + at, a.state_in && slot >= 0 ? 1 : 0, P * N * 4);
    const Rows out = rows_at(a.state_out + at, a.state_out && slot >= 0 ? 1 : 0, P * N * 4);
    auto offset = [&](int u, int i) -> uint32_t {                   // rows beyond the head are beyond its bytes
        const int n = at_n + i * V * lpr;
        return n < N ? (uint32_t)((p0 + u * rows) * N + n) * 4 : kOutside;
    };
    vec h[U][CI];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < CI; ++i) {
            if constexpr (V == 4) h[u][i] = __builtin_bit_cast(vec, __builtin_amdgcn_raw_buffer_load_b128(in, offset(u, i), 0, kStream));
            else h[u][i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(in, offset(u, i), 0, kStream));
        }
    const uint32_t e = sizeof(T);
    const int group = head / (a.heads / a.groups);
    const Rows brows = rows_at(a.b + (int64_t)first * a.b_stride + group * N, 1, N * e);
    const Rows crows = rows_at(a.c + (int64_t)first * a.c_stride + group * N, 1, N * e);
    const Rows xrows = rows_at(a.x + (int64_t)first * a.x_stride + (int64_t)head * P, 1, P * e);
    const Rows zrows = rows_at(a.z + (int64_t)first * a.z_stride + (int64_t)head * P, a.z ? 1 : 0, P * e);
    const Rows yrows = rows_at(a.y + (int64_t)first * a.y_stride + (int64_t)head * P, 1, P * e);
    float delta = (float)a.dt[(int64_t)first * a.dt_stride + head] + (a.dt_bias ? a.dt_bias[head] : 0.0f);
    Piece<T, V> b[CI], c[CI];
#pragma unroll
    for (int i = 0; i < CI; ++i) {
        const int n = at_n + i * V * lpr;
        b[i].template load<V == 4>(brows, n * e, N - n);
        c[i].template load<V == 4>(crows, n * e, N - n);
    }
    Piece<T, 1> x[U], z[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        x[u].template load<false>(xrows, (p0 + u * rows) * e, 1);
        z[u].template load<false>(zrows, (p0 + u * rows) * e, 1);
    }
    if (a.softplus) delta = softplus(delta);
    const float keep = expf(delta * a.a[head]), skip = a.d_skip ? a.d_skip[head] : 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const float in_x = delta * (float)x[u].v[0];
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < CI; ++i) {
            const bool has_n = at_n + i * V * lpr < N;              // (elsewhere infinities would meet zeros)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                h[u][i][k] = keep * h[u][i][k] + in_x * (float)b[i].v[k];
                s = has_n ? fmaf(h[u][i][k], (float)c[i].v[k], s) : s;
            }
            if constexpr (V == 4) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, h[u][i]), out, offset(u, i), 0, kStream);
            else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, (float)h[u][i][0]), out, offset(u, i), 0, kStream);
        }
        for (int m = lpr >> 1; m > 0; m >>= 1) s += __shfl_xor(s, m);
        if (a.d_skip) s += skip * (float)x[u].v[0];
        if (a.z) s *= silu_as<T>((float)z[u].v[0]);
        Piece<T, 1> y;
        y.v[0] = (T)s;
        y.template store<false>(yrows, (p0 + u * rows) * e, at_n == 0 ? 1 : 0);
    }
}

template <typename T> static int launch_step(const SsmArgs<T> &a, bool vec_bc, int sequences, hipStream_t st)
{
    const int V = a.vec_state && vec_bc ? 4 : 1;
    int lpr_log = 0;
    while (lpr_log < 6 && (V << lpr_log) < a.state_dim) ++lpr_log;
    const int rows = 256 >> lpr_log;
    // eight rows a lane keep enough bytes in flight; two where that would leave compute units without work
    const int64_t wide = (int64_t)a.heads * sequences * ((a.head_dim + 8 * rows - 1) / (8 * rows));
    const int U = wide >= 4 * kComputeUnits ? 8 : 2;
    const dim3 grid(a.heads, sequences, (a.head_dim + U * rows - 1) / (U * rows));
#define WPK_STEP(V, CI)                                                                                                \
    do {                                                                                                               \
        if (U == 8) hipLaunchKernelGGL((ssm_step_kernel<T, V, CI, 8>), grid, dim3(256), 0, st, a, lpr_log);            \
        else hipLaunchKernelGGL((ssm_step_kernel<T, V, CI, 2>), grid, dim3(256), 0, st, a, lpr_log);                   \
    } while (0)
    if (V == 4) WPK_STEP(4, 1);
    else if (a.state_dim <= 64) WPK_STEP(1, 1);
    else WPK_STEP(1, 4);
#undef WPK_STEP
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

// ---- prompts -----------------------------------------------------------------------------------------------
static const int kResidents = 2;      // workgroups that share a compute unit (most types and sizes)
static const int kPartUnit = 64;      // tokens that parts are multiples of: whole chunks of every kernel
struct ScanShape {
    int n_parts, part_units;
    bool by_length;           // requests of different lengths that do not all start at once: the longest first
};

// Requests are cut along their tokens where their heads alone would leave compute units idle, or where the longest one would
// still be walked through when the others are long done.  Every part but a request's last is walked through twice, first
// for the state that it leaves and then for y, which costs half as much again.  Heads of 64 x 128 numbers, bf16, calls whole and
// cut in turn: one request of 16384 tokens (32 heads) 1078 and 177 us, of 2048 138 and 42, of 512 38 and 33; 24 uneven ones, 12000
// tokens together, the longest 3833 (64 heads), 274 and 232; eight of 250 beside one of 3000 (32 heads) 209 and 68.  24 even ones
// (64 heads) stay whole: 170.
static ScanShape scan_shape(const wpk_ssm_desc &d)
{
    const int64_t units = (longest_request(d.tokens, d.max_length) + kPartUnit - 1) / kPartUnit;
    const int64_t teams = (int64_t)d.heads * ((d.head_dim + 63) / 64), room = kResidents * kComputeUnits;
    ScanShape s = {1, (int)units, teams * d.sequences > room && d.sequences > 1 && d.sequences <= 256};
    if (d.sequences == 0) return s;
    // units for each workgroup that runs at once, were they dealt out evenly
    const int64_t all = d.tokens / kPartUnit + (d.sequences + 1) / 2, share = (all * teams + room - 1) / room;
    if (units < 8 || units <= 2 * share) return s;
    int64_t each = share < 4 ? 4 : share;
    // (at most a GiB of workspace)
    int64_t most = (1ll << 30) / ((int64_t)d.sequences * d.heads * d.head_dim * d.state_dim * (int64_t)sizeof(float));
    if (most > 32) most = 32;
    if (most < 2) return s;
    if ((units + each - 1) / each > most) each = (units + most - 1) / most;
    s.n_parts = (int)((units + each - 1) / each);
    s.part_units = (int)each;
    return s;
}

static size_t scan_part_bytes(const wpk_ssm_desc &d, const ScanShape &s)
{
    return (size_t)d.sequences * d.heads * s.n_parts * d.head_dim * d.state_dim * sizeof(float);
}

template <typename T, int NPAD, int Q, bool WIDE> static int launch_scan_rows(SsmArgs<T> a, int sequences, hipStream_t st)
{
    a.part_chunks *= kPartUnit / Q;
    const unsigned heads = a.heads * ((a.head_dim + 63) / 64);
    if (a.n_parts > 1) {
        hipLaunchKernelGGL((ssm_scan_kernel<T, NPAD, Q, false, WIDE>), dim3(heads, a.n_parts - 1, sequences), dim3(256), 0, st, a);
        WPK_HIP(hipGetLastError());
        if (a.n_parts > 2) {
            const dim3 grid((a.head_dim * a.state_dim + 1023) / 1024, a.heads, sequences);
            hipLaunchKernelGGL((ssm_join_kernel<T, Q>), grid, dim3(256), 0, st, a);
            WPK_HIP(hipGetLastError());
        }
    }
    hipLaunchKernelGGL((ssm_scan_kernel<T, NPAD, Q, true, WIDE>), dim3(heads, a.n_parts, sequences), dim3(256), 0, st, a);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

// Chunks of 64 tokens where two workgroups of them fit a compute unit, else of 32: 32 heads of 64 numbers, 16384 tokens,
// bf16, states of 128: 155 us by 64 and 183 by 32; of 256: 313 and 344; f16, of 64: 157 and 179; of 128: 277 and 243.  But a
// workgroup that has its compute unit to itself gains nothing by smaller ones, f16: 10 heads of 48 x 72, 9 requests of 1001
// tokens together, 32.5 us by 64 and 36.9 by 32; states of 64 x 128, 1000 tokens of 64 heads, 50 and 55; 8192 of 4 heads, 55 and
// 60; 8 requests of 400 of 32 heads, 49 and 51, of 64, 12.6 both.  Rows that are moved element by element take more registers:
// bf16, of 128: 543 and 357; of 256: 1017 and 792 (its kernels for 16 bits keep some 40 registers in scratch memory, at two
// workgroups a compute unit).
template <typename T, int NPAD> static int launch_scan(const SsmArgs<T> &a, int sequences, hipStream_t st)
{
    const int Q = sizeof(T) == 4 || (SsmType<T>::parts == 2 && NPAD > 64) ? 32 : 64;
    if (!a.vec_rows) return launch_scan_rows<T, NPAD, 32, false>(a, sequences, st);
    if constexpr (SsmType<T>::parts == 2 && NPAD == 128) {
        const int64_t workgroups = (int64_t)sequences * a.heads * ((a.head_dim + 63) / 64) * a.n_parts;
        if (workgroups <= kComputeUnits) return launch_scan_rows<T, NPAD, 64, true>(a, sequences, st);
    }
    return launch_scan_rows<T, NPAD, Q, true>(a, sequences, st);
}

template <typename T> static int launch_scan(const SsmArgs<T> &a, int sequences, hipStream_t st)
{
    if (a.state_dim <= 32) return launch_scan<T, 32>(a, sequences, st);
    if (a.state_dim <= 64) return launch_scan<T, 64>(a, sequences, st);
    if (a.state_dim <= 128) return launch_scan<T, 128>(a, sequences, st);
    return launch_scan<T, 256>(a, sequences, st);
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
        d.state_dim > kMaxStateDim || d.sequences > 65535 || d.tokens > kMostRows || d.heads > 65535 || d.x_stride >= most || d.dt_stride >= most ||
        d.b_stride >= most || d.c_stride >= most || d.z_stride >= most || d.y_stride >= most)
        return WPK_E_UNSUPPORTED;
    return WPK_OK;
}

template <typename T>
static int ssm_typed(const wpk_ssm_desc &d, bool step, const void *x, const void *dt, const float *a, const void *b, const void *c,
                     const float *d_skip, const void *z, const float *dt_bias, const Requests &rq, const float *state_in,
                     float *state_out, void *y, void *workspace, hipStream_t st)
{
    // buffer accesses of up to 16 bytes want multiples of four
    auto rows_ok = [&](const void *p, int64_t stride) { return stride * (int64_t)sizeof(T) % 4 == 0 && aligned_to(p, 4); };
    ScanShape shape = scan_shape(d);
    if (!rq.starts) shape.by_length = false;
    SsmArgs<T> args = {(const T *)x, (const T *)dt, (const T *)b, (const T *)c, (const T *)z, a, d_skip, dt_bias, state_in,
                       state_out, (T *)y, rq, d.heads, d.head_dim, d.groups, d.state_dim, d.dt_softplus,
                       d.x_stride, d.dt_stride, d.b_stride, d.c_stride, d.z_stride, d.y_stride,
                       nullptr, nullptr, shape.n_parts, shape.part_units, shape.by_length ? d.sequences : 0,
                       d.state_dim % 8 == 0 && d.head_dim % 8 == 0 && rows_ok(b, d.b_stride) && rows_ok(c, d.c_stride) &&
                           rows_ok(x, d.x_stride) && (!z || rows_ok(z, d.z_stride)) && rows_ok(y, d.y_stride),
                       d.state_dim % 4 == 0 && aligned_to(state_in, 16) && aligned_to(state_out, 16)};
    if (step) return launch_step<T>(args, rows_ok(b, d.b_stride) && rows_ok(c, d.c_stride), d.sequences, st);
    if (shape.n_parts > 1) {
        args.parts = (float *)workspace;
        args.part_decay = (float *)((char *)workspace + scan_part_bytes(d, shape));
    }
    return launch_scan<T>(args, d.sequences, st);
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
    if (!step) {
        if (wpk_ssm_workspace_bytes(dp) > 0 && !workspace) return WPK_E_NULL_PTR;
        if (!aligned_to(workspace, 16)) return WPK_E_BAD_ARG;
    }
    const Requests rq = {starts, slot_map, resume, d.tokens, d.max_length, d.slots};
    const hipStream_t st = (hipStream_t)stream;
    if (d.dtype == WPK_BF16) return ssm_typed<bf16>(d, step, x, dt, a, b, c, d_skip, z, dt_bias, rq, state_in, state_out, y, workspace, st);
    if (d.dtype == WPK_F16) return ssm_typed<f16>(d, step, x, dt, a, b, c, d_skip, z, dt_bias, rq, state_in, state_out, y, workspace, st);
    return ssm_typed<float>(d, step, x, dt, a, b, c, d_skip, z, dt_bias, rq, state_in, state_out, y, workspace, st);
}

}  // namespace wpk

extern "C" {

int64_t wpk_ssm_workspace_bytes(const wpk_ssm_desc *d)
{
    const int rc = wpk::check_ssm(d);
    if (rc != WPK_OK) return rc;
    const wpk::ScanShape s = wpk::scan_shape(*d);
    if (s.n_parts < 2) return 0;
    return (int64_t)(wpk::scan_part_bytes(*d, s) + (size_t)d->sequences * d->heads * s.n_parts * sizeof(float));
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
