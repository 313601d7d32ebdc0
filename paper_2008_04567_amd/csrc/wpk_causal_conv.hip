// Short causal convolution of every channel by itself, over ragged requests that carry a state.
//
// y[t][c] = act(bias[c] + sum_j w[c][j] x[t - (W-1) + j][c]).  Bound by memory: every value is read once and written
// once for W multiply-adds.  A lane owns V channels (16 bytes where rows start at multiples of four) and a run of kRun tokens: it
// keeps the last W - 1 rows in registers, so rows are read W - 1 times more than once per run only, and asks for kAhead
// rows at once.  16384 ragged tokens of 4352 bf16 channels: 62 us, 4.6 TB/s, the kernel alone, and 68 (4.2 TB/s) a call behind
// others (before its weights were read by vectors, 66 alone; so measured, runs of 16 took 67, four rows at once 72, two 80).
#include "wpk_seq.h"

namespace wpk {

static const int kRun = 32;   // tokens of a run
static const int kAhead = 8;  // rows under way

template <typename T, int V> struct Row {
    typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));      // (the device takes such loads and stores)
};

template <typename T, int V> __device__ inline void load_row(const T *p, float (&out)[V])
{
    const typename Row<T, V>::vec a = *(const typename Row<T, V>::vec *)p;
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = (float)a[i];
}

// but for the first `skip`
template <typename T, int V> __device__ inline void store_row(T *p, typename Row<T, V>::vec v, int skip)
{
    if (skip == 0) {
        *(typename Row<T, V>::vec *)p = v;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i >= skip) p[i] = v[i];
    }
}

template <typename T> struct ConvArgs {
    const T *x, *w, *bias, *state_in;
    T *state_out, *y;
    Requests rq;
    int32_t channels, lanes, runs, act;   // lanes: of one run; runs: of a request of max_length
    int64_t x_stride, y_stride;
};

// Grid: (lanes of all runs / 256, requests).  Rows before a request's first come from its state; the lane of the first
// run also writes the state that the request leaves, after it has read the old one, so the two may be the same.  The last
// lane of a row takes the row's last V channels and stores those that no lane before it has.
template <typename T, int V, int W> __global__ void __launch_bounds__(256) causal_conv_kernel(ConvArgs<T> a)
{
    const int lane = blockIdx.x * 256 + threadIdx.x;
    int run = lane / a.lanes;
    if (run >= a.runs) return;
    const int c_first = (lane - run * a.lanes) * V, c = min(c_first, a.channels - V), skip = c_first - c;
    int first, length;
    request_rows(a.rq, blockIdx.y, &first, &length);
    const bool head = run == 0;
    if (!head && run * kRun >= length) return;

    float w[W][V], b[V], win[W][V];
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = 0.0f;
    if (a.bias) load_row<T, V>(a.bias + c, b);
#pragma unroll
    for (int k = 0; k < W; ++k) {             // the lane's V W weights stand one after another
        float part[V];
        load_row<T, V>(a.w + (size_t)c * W + k * V, part);
#pragma unroll
        for (int i = 0; i < V; ++i) w[(k * V + i) % W][(k * V + i) / W] = part[i];
    }
    const T *x = a.x + (int64_t)first * a.x_stride + c;
    T *y = a.y + (int64_t)first * a.y_stride + c;

    if (head) {
        const int slot = request_slot(a.rq, blockIdx.y);
        const bool resume = a.state_in && slot >= 0 && request_resumes(a.rq, blockIdx.y);
        const size_t at = (size_t)max(slot, 0) * (W - 1) * a.channels + c;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            if (resume) load_row<T, V>(a.state_in + at + (size_t)j * a.channels, win[j]);
            else
#pragma unroll
                for (int i = 0; i < V; ++i) win[j][i] = 0.0f;
        }
        if (a.state_out && slot >= 0) {
#pragma unroll
            for (int j = 0; j < W - 1; ++j) {      // row j of the new state is row length + j of [old state | x]
                float r[V];
                typename Row<T, V>::vec left;
                const int row = length - (W - 1) + j;
                if (row >= 0) load_row<T, V>(x + (int64_t)row * a.x_stride, r);
                else {
#pragma unroll
                    for (int i = 0; i < V; ++i) r[i] = 0.0f;
#pragma unroll
                    for (int o = 0; o < W - 1; ++o)
                        if (o == length + j)
#pragma unroll
                            for (int i = 0; i < V; ++i) r[i] = win[o][i];
                }
#pragma unroll
                for (int i = 0; i < V; ++i) left[i] = (T)r[i];
                store_row<T, V>(a.state_out + at + (size_t)j * a.channels, left, skip);
            }
        }
    }
    // requests longer than max_length go on with their next runs
    for (; run * kRun < length; run += a.runs) {
        const int t0 = run * kRun, t1 = min(t0 + kRun, length);
        if (run > 0) {
#pragma unroll
            for (int j = 0; j < W - 1; ++j) load_row<T, V>(x + (int64_t)(t0 - (W - 1) + j) * a.x_stride, win[j]);
        }
        // kAhead rows are asked for at once; rows behind the run are read as its last one and not used
        for (int t = t0; t < t1; t += kAhead) {
            typename Row<T, V>::vec ahead[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) ahead[u] = *(const typename Row<T, V>::vec *)(x + (int64_t)min(t + u, t1 - 1) * a.x_stride);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                typename Row<T, V>::vec out;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    win[W - 1][i] = (float)ahead[u][i];
                    float s = b[i];
#pragma unroll
                    for (int j = 0; j < W; ++j) s = fmaf(w[j][i], win[j][i], s);
                    out[i] = (T)(a.act == WPK_ACT_SILU ? silu_as<T>(s) : s);
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) win[j][i] = win[j + 1][i];
                }
                if (t + u < t1) store_row<T, V>(y + (int64_t)(t + u) * a.y_stride, out, skip);
            }
        }
    }
}

template <typename T, int V, int W> static int launch_conv(const ConvArgs<T> &a, int sequences, hipStream_t st)
{
    const dim3 grid((unsigned)(((int64_t)a.lanes * a.runs + 255) / 256), sequences);
    hipLaunchKernelGGL((causal_conv_kernel<T, V, W>), grid, dim3(256), 0, st, a);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

template <typename T, int V> static int launch_conv_width(const ConvArgs<T> &a, int width, int sequences, hipStream_t st)
{
    switch (width) {
    case 2: return launch_conv<T, V, 2>(a, sequences, st);
    case 3: return launch_conv<T, V, 3>(a, sequences, st);
    case 4: return launch_conv<T, V, 4>(a, sequences, st);
    case 5: return launch_conv<T, V, 5>(a, sequences, st);
    case 6: return launch_conv<T, V, 6>(a, sequences, st);
    case 7: return launch_conv<T, V, 7>(a, sequences, st);
    default: return launch_conv<T, V, 8>(a, sequences, st);
    }
}

template <typename T>
static int conv_typed(const wpk_causal_conv_desc &d, const void *x, const void *w, const void *bias, const Requests &rq,
                      const void *state_in, void *state_out, void *y, hipStream_t st)
{
    // 16 bytes of channels a lane where every row starts at a multiple of four, else one channel: 16384 tokens of 4348 bf16
    // channels take 72 us by 16 bytes and 90 by one; rows at odd multiples of two gain in large calls only (4351 channels: 76
    // and 90) and lose in others (2000 tokens of 1763: 17.7 and 9.6)
    const int V = 16 / (int)sizeof(T);
    auto fours = [](const void *p, int64_t stride) { return aligned_to(p, 4) && stride * (int64_t)sizeof(T) % 4 == 0; };
    const bool wide = d.channels >= V && fours(x, d.x_stride) && fours(y, d.y_stride) && fours(w, 0) && fours(bias, 0) &&
                      fours(state_in, d.channels) && fours(state_out, d.channels);
    ConvArgs<T> a = {(const T *)x, (const T *)w, (const T *)bias, (const T *)state_in, (T *)state_out, (T *)y, rq,
                     d.channels, wide ? (d.channels + V - 1) / V : d.channels,
                     (longest_request(d.tokens, d.max_length) + kRun - 1) / kRun, d.act, d.x_stride, d.y_stride};
    // (a lane's number has 31 bits: a request of more runs than that is done by lanes that take several)
    const int64_t most = 0x40000000 / a.lanes;
    if (a.runs > most) a.runs = (int32_t)(most < 1 ? 1 : most);
    return wide ? launch_conv_width<T, V>(a, d.width, d.sequences, st) : launch_conv_width<T, 1>(a, d.width, d.sequences, st);
}

static int conv_call(const wpk_causal_conv_desc *dp, bool step, const void *x, const void *w, const void *bias,
                     const int32_t *starts, const int32_t *slot_map, const int32_t *resume, const void *state_in,
                     void *state_out, void *y, void *stream)
{
    if (!dp) return WPK_E_NULL_PTR;
    const wpk_causal_conv_desc d = *dp;
    if (d.sequences < 0 || d.tokens < 0 || d.max_length < 1 || d.channels < 1 || d.width < 2 || d.slots < 0 ||
        d.x_stride < d.channels || d.y_stride < d.channels)
        return WPK_E_BAD_DESC;
    if (!seq_type_ok(d.dtype) || (d.act != WPK_ACT_NONE && d.act != WPK_ACT_SILU) || d.width > 8 ||
        d.sequences > 65535 || d.tokens > kMostRows || d.channels > 0x3fffffff || d.x_stride >= (1ll << 40) || d.y_stride >= (1ll << 40))
        return WPK_E_UNSUPPORTED;
    const size_t e = seq_type_bytes(d.dtype);
    int rc = check_requests(d.sequences, d.tokens, d.max_length, d.slots, step, starts, slot_map, resume, state_in, state_out, e);
    if (rc != WPK_OK) return rc;
    if (d.sequences == 0) return WPK_OK;
    if (!w || (d.tokens > 0 && (!x || !y))) return WPK_E_NULL_PTR;
    if (!aligned_to(x, e) || !aligned_to(w, e) || !aligned_to(bias, e) || !aligned_to(y, e)) return WPK_E_BAD_ARG;
    const Requests rq = {starts, slot_map, resume, d.tokens, d.max_length, d.slots};
    const hipStream_t st = (hipStream_t)stream;
    if (d.dtype == WPK_BF16) return conv_typed<bf16>(d, x, w, bias, rq, state_in, state_out, y, st);
    if (d.dtype == WPK_F16) return conv_typed<f16>(d, x, w, bias, rq, state_in, state_out, y, st);
    return conv_typed<float>(d, x, w, bias, rq, state_in, state_out, y, st);
}

}  // namespace wpk

extern "C" {

int wpk_causal_conv1d_fwd(const wpk_causal_conv_desc *d, const void *x, const void *w, const void *bias, const int32_t *starts,
                          const int32_t *slot_map, const int32_t *resume, const void *state_in, void *state_out, void *y,
                          void *stream)
{
    return wpk::conv_call(d, false, x, w, bias, starts, slot_map, resume, state_in, state_out, y, stream);
}

int wpk_causal_conv1d_step(const wpk_causal_conv_desc *d, const void *x, const void *w, const void *bias,
                           const int32_t *slot_map, const void *state_in, void *state_out, void *y, void *stream)
{
    return wpk::conv_call(d, true, x, w, bias, nullptr, slot_map, nullptr, state_in, state_out, y, stream);
}

}  // extern "C"
