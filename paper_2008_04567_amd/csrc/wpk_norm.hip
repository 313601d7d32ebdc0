// RMS norm with the residual's addition, and rows in 8 bits.
//
// Both are passes over memory (bound: its bytes; for few rows, a launch and two latencies).  A lane holds eight neighbouring
// elements at a time, so a block of 128 values that share a scale is a row of 16 lanes, and its largest magnitude is found
// without LDS.
#include <type_traits>

#include "wpk_q8.h"

namespace wpk {

struct NormArgs {
    const void *x, *residual, *gain;
    const int32_t *source;
    const float *weights;
    void *h, *y;
    uint8_t *q;
    float *scales;
    int32_t rows, width, groups, parts, x_rows;      // width: of a group
    float eps;
    int64_t x_stride, residual_stride, h_stride, y_stride, q_stride, scale_stride;
};

// the number of this workgroup, in a grid of two dimensions
__device__ inline int64_t workgroup() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// LANES lanes to a row (of one group), P pieces of eight elements each lane; a workgroup of 256 threads has several rows where
// LANES is 64.  ALL: a row is LANES * P * 8 elements exactly.  A row stays in registers between the sum of its squares and the
// result, so every input is read once; parts of a row are asked for four at a time.  16384 x 4096 bf16 with residual, into h and 8
// bits: 87 us, 5.4 TB/s (a copy reaches 5.1); eight parts for each of 4096 rows of 2048: 32 us, 5.8 TB/s; 16 rows of 2048: 3.0 us,
// of which a launch is most.
// Rows beyond 32768 (P = 8) keep 40 to 50 registers in scratch memory, 16-bit ones of exactly 65536 columns 126.
template <typename T, int LANES, int P, bool ALL, bool FAR> __global__ void __launch_bounds__(LANES < 256 ? 256 : LANES) rms_norm_kernel(NormArgs a)
{
    const int kWaves = LANES / 64;
    const bool kLong = P > 2;         // rows that take most registers: a part and a piece at a time, the gain when it is needed
    const int lane = threadIdx.x % LANES;
    const int64_t units = (int64_t)a.rows * a.groups;
    int64_t unit = workgroup();
    if (LANES == 64) {
        unit = unit * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    }
    if (unit >= units) return;
    const int64_t row = a.groups == 1 ? unit : unit / a.groups;
    const int c0 = a.groups == 1 ? 0 : (int)(unit - row * a.groups) * a.width;

    f32x8 s[P];
    int left[P], at[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int c = (lane + LANES * p) * 8;
        left[p] = a.width - c;
        at[p] = c0 + c;
    }
    auto row_of = [&](const void *base, int64_t stride, int64_t r, int p) { return (const T *)base + r * stride + at[p]; };
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (a.residual) s[p] = Eight<T>::template load<ALL, false>(row_of(a.residual, a.residual_stride, row, p), left[p]);
        else s[p] = f32x8{0, 0, 0, 0, 0, 0, 0, 0};
    }
    if (a.parts == 1 && !a.source) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            f32x8 v = Eight<T>::template load<ALL, FAR>(row_of(a.x, a.x_stride, row, p), left[p]);
            if (a.weights) v *= a.weights[row];
            s[p] += v;
        }
    } else {
        // a row that is not there is read as one that is, and counts as zeros
        auto add = [&](auto number, int j0) {
            const int N = decltype(number)::value;             // parts under way at a time
            f32x8 v[N][P];
            float w[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int64_t e = row * a.parts + j0 + j;
                const int64_t from = a.source ? a.source[e] : e;
                const bool there = from >= 0 && from < a.x_rows;
                w[j] = there ? (a.weights ? a.weights[e] : 1.0f) : 0.0f;
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    if constexpr (kLong) {
                        const f32x8 u = Eight<T>::template load<ALL, FAR>(row_of(a.x, a.x_stride, there ? from : 0, p), left[p]);
                        if (there) s[p] += u * w[j];
                        __builtin_amdgcn_sched_barrier(0);
                        continue;
                    }
                    v[j][p] = Eight<T>::template load<ALL, FAR>(row_of(a.x, a.x_stride, there ? from : 0, p), left[p]);
                    if (!there) v[j][p] = f32x8{0, 0, 0, 0, 0, 0, 0, 0};
                }
            }
            if constexpr (kLong) return;
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int p = 0; p < P; ++p) s[p] += v[j][p] * w[j];
        };
        int j0 = 0;
        if constexpr (!kLong) {
            for (; j0 + 4 <= a.parts; j0 += 4) add(std::integral_constant<int, 4>(), j0);
            if (a.parts - j0 >= 2) add(std::integral_constant<int, 2>(), j0), j0 += 2;
        }
        for (; j0 < a.parts; ++j0) add(std::integral_constant<int, 1>(), j0);
    }
    auto gain_of = [&](int p) {
        return a.gain ? Eight<T>::template load<ALL, false>((const T *)a.gain + at[p], left[p]) : f32x8{1, 1, 1, 1, 1, 1, 1, 1};
    };
    f32x8 gain[kLong ? 1 : P];
    if constexpr (!kLong)
#pragma unroll
        for (int p = 0; p < P; ++p) gain[p] = gain_of(p);
    __shared__ float part[2][kWaves];
    auto squares = [&](float by, int turn) {                   // sum of (by s)^2 over the row
        float sum = 0.0f;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const f32x8 u = s[p] * by, e = u * u;
            sum += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
        }
        sum = wave_total(sum);
        if (kWaves > 1) {
            if ((lane & 63) == 0) part[turn][lane >> 6] = sum;
            __syncthreads();
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) sum += part[turn][i];
        }
        return sum;
    };
#pragma unroll
    for (int p = 0; p < P; ++p)
        if (a.h && (ALL || left[p] > 0)) Eight<T>::template store<ALL, FAR>((T *)a.h + row * a.h_stride + at[p], left[p], s[p]);
    const float sum = squares(1.0f, 0);
    float r = rsqrtf(sum / (float)a.width + a.eps);
    // Squares that are no 32-bit numbers, or no normal ones where eps does not hide them, are formed again of scaled values.  The
    // scale and the root stay two factors, since the reciprocal root of the whole may be no 32-bit number itself (above 2^128 for
    // rows of the smallest numbers, below 2^-126 for those of the largest), in the order in which no product leaves the range:
    // values grow before they meet the root, or meet it before they shrink.
    const float by = sum > 3.4e38f ? 0x1p-80f : sum < 0x1p-90f && a.eps < 0x1p-90f ? 0x1p100f : 1.0f;
    if (by != 1.0f) {
        const float root = rsqrtf(squares(by, 1) / (float)a.width + a.eps * by * by), first = by > 1.0f ? by : root;
        r = by > 1.0f ? root : by;
#pragma unroll
        for (int p = 0; p < P; ++p) s[p] *= first;
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if constexpr (kLong) {
            gain[0] = gain_of(p);
            __builtin_amdgcn_sched_barrier(0);
        }
        const f32x8 v = s[p] * r * gain[kLong ? 0 : p];
        if (a.y && (ALL || left[p] > 0)) Eight<T>::template store<ALL, FAR>((T *)a.y + row * a.y_stride + at[p], left[p], v);
        // (a row's last block: the lanes behind it hold zeros)
        if (a.q) store_8<ALL, FAR>(a.q + row * a.q_stride + at[p], a.scales + row * a.scale_stride + at[p] / kScaleBlock, left[p], v, lane % 16 == 0);
    }
}

struct QuantizeArgs {
    const void *x;
    uint8_t *q;
    float *scales;
    int32_t rows, width, blocks, shift;     // blocks of a row; a workgroup's 16 blocks at a time are 16 >> shift rows of 1 << shift
    int64_t x_stride, q_stride, scale_stride;
};

// 16 lanes to a block, U blocks a lane under way: as many as a row has, up to 64.  16384 x 4096 bf16: 35 us, 5.8 TB/s (with twice the U
// that rows of 32 blocks fill, 47); 1777 x 1544 f16: 4.0 us (7.5 with U = 4).
template <typename T, int U, bool FAR> __global__ void __launch_bounds__(256) quantize_kernel(QuantizeArgs a)
{
    const int unit = threadIdx.x >> 4, lane = threadIdx.x & 15, rows = 16 >> a.shift;
    const int in_row = unit & ((1 << a.shift) - 1);
    const int64_t row0 = workgroup() * (a.shift == 4 ? 1 : rows * U) + (unit >> a.shift);
    // either U rows of up to 16 blocks, or one row U times 16 blocks at a time
    for (int b0 = 0; b0 < a.blocks; b0 += 16 * U) {
        f32x8 v[U];
        int left[U];
        int64_t row[U], c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            row[u] = a.shift == 4 ? row0 : row0 + u * rows;
            c[u] = ((int64_t)(a.shift == 4 ? b0 + 16 * u : 0) + in_row) * kScaleBlock + lane * 8;
            left[u] = row[u] < a.rows && c[u] < a.width ? (int)min((int64_t)a.width - c[u], (int64_t)8) : 0;
            v[u] = f32x8{0, 0, 0, 0, 0, 0, 0, 0};
            if (left[u] > 0) v[u] = Eight<T>::template load<false, FAR>((const T *)a.x + row[u] * a.x_stride + c[u], left[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            store_8<false, FAR>(a.q + row[u] * a.q_stride + c[u], a.scales + row[u] * a.scale_stride + c[u] / kScaleBlock, left[u], v[u],
                           lane == 0);
        if (a.shift < 4) break;
    }
}

static bool stride_ok(int64_t stride, int64_t least, int64_t most, int *rc)
{
    if (stride < least) *rc = WPK_E_BAD_DESC;
    else if (stride >= most) *rc = WPK_E_UNSUPPORTED;
    return *rc == WPK_OK;
}

// Workgroups `n` in two dimensions, since threads in one are fewer than 2^32.
static dim3 grid_of(int64_t n) { return n <= 1 << 20 ? dim3((unsigned)n) : dim3(1 << 20, (unsigned)((n + (1 << 20) - 1) >> 20)); }

template <typename T, int LANES, int P> static void launch_norm(const NormArgs &a, hipStream_t st)
{
    const int64_t units = (int64_t)a.rows * a.groups;
    const dim3 grid = grid_of(LANES == 64 ? (units + 3) / 4 : units), block(LANES < 256 ? 256 : LANES);
    const bool all = a.width == LANES * P * 8, far = units * a.width * (a.parts + 1) * (int64_t)sizeof(T) > kFarBytes;
    if (all && far) hipLaunchKernelGGL((rms_norm_kernel<T, LANES, P, true, true>), grid, block, 0, st, a);
    else if (all) hipLaunchKernelGGL((rms_norm_kernel<T, LANES, P, true, false>), grid, block, 0, st, a);
    else if (far) hipLaunchKernelGGL((rms_norm_kernel<T, LANES, P, false, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((rms_norm_kernel<T, LANES, P, false, false>), grid, block, 0, st, a);
}

template <typename T> static int norm_typed(const NormArgs &a, hipStream_t st)
{
    const int w = a.width;
    if (w <= 512) launch_norm<T, 64, 1>(a, st);
    else if (w <= 1024) launch_norm<T, 64, 2>(a, st);
    else if (w <= 2048) launch_norm<T, 256, 1>(a, st);
    else if (w <= 4096) launch_norm<T, 256, 2>(a, st);
    else if (w <= 8192) launch_norm<T, 1024, 1>(a, st);
    else if (w <= 16384) launch_norm<T, 1024, 2>(a, st);
    else if (w <= 32768) launch_norm<T, 1024, 4>(a, st);
    else launch_norm<T, 1024, 8>(a, st);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

template <typename T, int U> static int launch_quantize(const QuantizeArgs &a, hipStream_t st)
{
    const int64_t rows = a.shift == 4 ? 1 : (int64_t)(16 >> a.shift) * U;
    const dim3 grid = grid_of((a.rows + rows - 1) / rows);
    if ((int64_t)a.rows * a.width * (int64_t)sizeof(T) > kFarBytes) hipLaunchKernelGGL((quantize_kernel<T, U, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((quantize_kernel<T, U, false>), grid, dim3(256), 0, st, a);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

template <typename T> static int quantize_typed(const QuantizeArgs &a, hipStream_t st)
{
    if (a.shift == 4 && a.blocks <= 16) return launch_quantize<T, 1>(a, st);
    if (a.shift == 4 && a.blocks <= 32) return launch_quantize<T, 2>(a, st);
    return launch_quantize<T, 4>(a, st);
}

}  // namespace wpk

extern "C" {

int wpk_rms_norm_fwd(const wpk_rms_norm_desc *dp, const void *x, const int32_t *source, const float *weights,
                     const void *residual, const void *gain, void *h, void *y, void *q, float *scales, void *stream)
{
    using namespace wpk;
    if (!dp) return WPK_E_NULL_PTR;
    const wpk_rms_norm_desc d = *dp;
    const int64_t most = 1ll << 30;
    int rc = WPK_OK;
    if (d.rows < 0 || d.width < 1 || d.groups < 1 || d.parts < 1 || d.x_rows < 0 || d.width % d.groups != 0 || !(d.eps >= 0.0f))
        return WPK_E_BAD_DESC;
    if (d.rows > kMostRows || d.x_rows > kMostRows || d.width > 65536 || d.parts > 64 || !seq_type_ok(d.dtype)) return WPK_E_UNSUPPORTED;
    if (!stride_ok(d.x_stride, d.width, most, &rc) || !stride_ok(d.residual_stride, d.width, most, &rc) ||
        !stride_ok(d.h_stride, d.width, most, &rc) || !stride_ok(d.y_stride, d.width, most, &rc) ||
        !stride_ok(d.q_stride, d.width, most, &rc) || !stride_ok(d.scale_stride, scale_blocks(d.width), most, &rc))
        return rc;
    const int width = d.width / d.groups;
    if ((int64_t)d.rows * d.groups >= 1ll << 31) return WPK_E_UNSUPPORTED;
    if (d.q_stride % 16 != 0 || (q && d.groups > 1 && width % kScaleBlock != 0)) return WPK_E_UNSUPPORTED;
    if (d.rows == 0) return WPK_OK;
    if (!source && (int64_t)d.rows * d.parts > d.x_rows) return WPK_E_BAD_ARG;
    if (d.x_rows < 1) return WPK_E_BAD_ARG;
    if (!x || (!h && !y && !q) || (q && !scales)) return WPK_E_NULL_PTR;
    const size_t e = seq_type_bytes(d.dtype);
    if (!aligned_to(x, e) || !aligned_to(residual, e) || !aligned_to(gain, e) || !aligned_to(h, e) || !aligned_to(y, e) ||
        !aligned_to(q, 16) || !aligned_to(scales, 4) || !aligned_to(source, 4) || !aligned_to(weights, 4))
        return WPK_E_BAD_ARG;
    const NormArgs a = {x, residual, gain, source, weights, h, y, (uint8_t *)q, scales, d.rows, width, d.groups, d.parts, d.x_rows,
                        d.eps, d.x_stride, d.residual_stride, d.h_stride, d.y_stride, d.q_stride, d.scale_stride};
    const hipStream_t st = (hipStream_t)stream;
    if (d.dtype == WPK_BF16) return norm_typed<bf16>(a, st);
    if (d.dtype == WPK_F16) return norm_typed<f16>(a, st);
    return norm_typed<float>(a, st);
}

int wpk_quantize_fwd(const wpk_quantize_desc *dp, const void *x, void *q, float *scales, void *stream)
{
    using namespace wpk;
    if (!dp) return WPK_E_NULL_PTR;
    const wpk_quantize_desc d = *dp;
    const int64_t most = 1ll << 30;
    int rc = WPK_OK;
    if (d.rows < 0 || d.width < 1) return WPK_E_BAD_DESC;
    if (d.rows > kMostRows || d.width > kMostRows || !seq_type_ok(d.dtype) || d.reserved != 0) return WPK_E_UNSUPPORTED;
    if (!stride_ok(d.x_stride, d.width, most, &rc) || !stride_ok(d.q_stride, d.width, most, &rc) ||
        !stride_ok(d.scale_stride, scale_blocks(d.width), most, &rc))
        return rc;
    if (d.q_stride % 16 != 0) return WPK_E_UNSUPPORTED;
    if (d.rows == 0) return WPK_OK;
    if (!x || !q || !scales) return WPK_E_NULL_PTR;
    if (!aligned_to(x, seq_type_bytes(d.dtype)) || !aligned_to(q, 16) || !aligned_to(scales, 4)) return WPK_E_BAD_ARG;
    const int blocks = (int)scale_blocks(d.width);
    int shift = 0;
    while (shift < 4 && (1 << shift) < blocks) ++shift;
    const QuantizeArgs a = {x, (uint8_t *)q, scales, d.rows, d.width, blocks, shift, d.x_stride, d.q_stride, d.scale_stride};
    const hipStream_t st = (hipStream_t)stream;
    if (d.dtype == WPK_BF16) return quantize_typed<bf16>(a, st);
    if (d.dtype == WPK_F16) return quantize_typed<f16>(a, st);
    return quantize_typed<float>(a, st);
}

}  // extern "C"
