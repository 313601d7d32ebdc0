// Matrix product y = act(x w^T + bias) + residual.
//
// Three kernels share the work.  All of them multiply with w's rows as the MFMA's rows and x's as its columns, so a lane holds
// four neighbouring columns of one row of y at a time.
//   rows    few rows of x (a token of every request): w is streamed once, straight into registers, the reduction dealt out
//           to the waves of a workgroup (bound: w's bytes)
//   tiles   more rows: tiles of x and w through LDS (bound: the matrix pipes), in two forms: 16-bit operands in aligned rows
//           are loaded to LDS directly, others through registers
//   join    sums the partial products of workgroups that share an output along the reduction, in a fixed order
// fp32 is multiplied as such by the first, and as sums of three bf16 numbers by the second.
#include "wpk_seq.h"

namespace wpk {

struct LinearArgs {
    const void *x, *w, *bias, *residual;
    void *y;
    float *part;                      // partial products [slice][m][part_stride], where the reduction is cut
    int32_t m, n, k, act, y_f32;
    int32_t slices, slice_k;          // reduction entries of a slice (a multiple of 64)
    int32_t width;                    // columns of a workgroup of the row kernel (a multiple of four)
    int32_t wide_y;                   // rows of y (and the residual, the bias) hold whole aligned groups of four
    int64_t x_stride, w_stride, y_stride, residual_stride, part_stride;
};

template <typename T> struct Mma;
template <> struct Mma<bf16> {
    typedef bf16x8 v8;
    static __device__ f32x4 m16(v8 a, v8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ f32x16 m32(v8 a, v8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mma<f16> {
    typedef f16x8 v8;
    static __device__ f32x4 m16(v8 a, v8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ f32x16 m32(v8 a, v8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct Mma<float> {
    typedef f32x8 v8;
    // (the order of the reduction's entries does not matter as long as both operands have it: lane group g gives entry 8 g + j
    // to the j-th of eight steps of four)
    static __device__ f32x4 m16(v8 a, v8 b, f32x4 c)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
};

// eight neighbouring elements from an address that is aligned to one of them (the device takes such loads)
template <typename T> struct Octet {
    typedef T vec __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    static __device__ typename Mma<T>::v8 load(const T *p) { return *(const vec *)p; }
    static __device__ typename Mma<T>::v8 load_some(const T *p, int left)
    {
        typename Mma<T>::v8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : (T)0.0f;
        return v;
    }
};

// What follows the sums: columns n .. n + 3 of row m.
template <typename T, typename Y> __device__ inline void finish(const LinearArgs &a, int m, int n, f32x4 v)
{
    typedef T tvec __attribute__((ext_vector_type(4)));
    typedef Y yvec __attribute__((ext_vector_type(4)));
    if (m >= a.m || n >= a.n) return;
    Y *const y = (Y *)a.y + (int64_t)m * a.y_stride + n;
    const T *const r = (const T *)a.residual + (int64_t)m * a.residual_stride + n, *const b = (const T *)a.bias + n;
    if (a.wide_y) {
        if (a.bias) v += __builtin_convertvector(*(const tvec *)b, f32x4);
        v = apply_act<Y>(v, a.act);
        if (a.residual) v += __builtin_convertvector(*(const tvec *)r, f32x4);
        *(yvec *)y = __builtin_convertvector(v, yvec);
    } else {
        const int left = min(4, a.n - n);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (a.bias && i < left) v[i] += (float)b[i];
        v = apply_act<Y>(v, a.act);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) y[i] = (Y)(a.residual ? v[i] + (float)r[i] : v[i]);
    }
}
template <typename T> __device__ inline void finish(const LinearArgs &a, int m, int n, f32x4 v)
{
    if (sizeof(T) == 4 || a.y_f32) finish<T, float>(a, m, n, v);
    else finish<T, T>(a, m, n, v);
}
// ... or, where the reduction is cut, the partial sums
template <typename T> __device__ inline void finish_or_part(const LinearArgs &a, int slice, int m, int n, f32x4 v)
{
    if (a.slices == 1) finish<T>(a, m, n, v);
    else if (m < a.m && n < a.n) *(f32x4 *)(a.part + ((int64_t)slice * a.m + m) * a.part_stride + n) = v;
}

template <typename T> __global__ void __launch_bounds__(256) linear_join_kernel(LinearArgs a)
{
    const int quads = (a.n + 3) / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)quads * a.m) return;
    const int m = (int)(i / quads), n = (int)(i - (int64_t)m * quads) * 4;
    f32x4 v = {0, 0, 0, 0};
    for (int s = 0; s < a.slices; ++s) v += *(const f32x4 *)(a.part + ((int64_t)s * a.m + m) * a.part_stride + n);
    finish<T>(a, m, n, v);
}

// ---- few rows ------------------------------------------------------------------------------------------------
// A workgroup of eight waves owns `width` columns of y, 16 NT at most, and all of up to 16 MT rows.  A wave takes every eighth run
// of 64 reduction entries (a line of a row of w in 16-bit types) of its slice and keeps U of them in flight.  Rows beyond the
// matrices or the width are read as the last one (lines that are on their way already); nothing of them is stored.
// 32 rows by 8512 columns of 2048, bf16: 10.8 us, 3.3 TB/s of w; one row by 1024 columns: 4 us, of which a launch is most.
static const int kRowsWaves = 8;
template <typename T, int MT, int NT, int U> __global__ void __launch_bounds__(64 * kRowsWaves) linear_rows_kernel(LinearArgs a)
{
    typedef typename Mma<T>::v8 v8;
    __shared__ __align__(16) f32x4 sums[kRowsWaves][MT * NT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * a.width, n_end = min(n0 + a.width, a.n), slice = blockIdx.y;
    const int k_end = min(a.k, (slice + 1) * a.slice_k), k_begin = slice * a.slice_k + 64 * wave;
    const T *wp[NT], *xp[MT];
#pragma unroll
    for (int i = 0; i < NT; ++i) wp[i] = (const T *)a.w + (int64_t)min(n0 + 16 * i + row, n_end - 1) * a.w_stride + 8 * g;
#pragma unroll
    for (int i = 0; i < MT; ++i) xp[i] = (const T *)a.x + (int64_t)min(16 * i + row, a.m - 1) * a.x_stride + 8 * g;
    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

    v8 fw[U][2][NT], fx[U][2][MT];
    auto fetch = [&](int u, int k) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < NT; ++i) fw[u][h][i] = Octet<T>::load(wp[i] + k + 32 * h);
#pragma unroll
            for (int i = 0; i < MT; ++i) fx[u][h][i] = Octet<T>::load(xp[i] + k + 32 * h);
        }
    };
    auto multiply = [&](int u) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = Mma<T>::m16(fw[u][h][j], fx[u][h][i], acc[i][j]);
    };
    const int step = 64 * kRowsWaves;
    int k = k_begin;
    // U runs in flight: run u is asked for again as soon as it has been multiplied
    if (k + (U - 1) * step + 64 <= k_end) {
#pragma unroll
        for (int u = 0; u < U; ++u) fetch(u, k + u * step);
        for (; k + (2 * U - 1) * step + 64 <= k_end; k += U * step) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                multiply(u);
                fetch(u, k + (U + u) * step);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) multiply(u);
        k += U * step;
    }
    for (; k + 64 <= k_end; k += step) {
        fetch(0, k);
        multiply(0);
    }
    if (k < k_end) {                  // the reduction's last entries, fewer than 64
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int left = k_end - (k + 32 * h + 8 * g);
#pragma unroll
            for (int i = 0; i < NT; ++i) fw[0][h][i] = Octet<T>::load_some(wp[i] + k + 32 * h, left);
#pragma unroll
            for (int i = 0; i < MT; ++i) fx[0][h][i] = Octet<T>::load_some(xp[i] + k + 32 * h, left);
        }
        multiply(0);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) sums[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    for (int t = wave; t < MT * NT; t += kRowsWaves) {
        f32x4 v = sums[0][t][lane];
#pragma unroll
        for (int s = 1; s < kRowsWaves; ++s) v += sums[s][t][lane];
        const int n = n0 + 16 * (t % NT) + 4 * g;
        if (n < n_end) finish_or_part<T>(a, slice, 16 * (t / NT) + row, n, v);
    }
}

// ---- tiles -----------------------------------------------------------------------------------------------------
// Workgroups are dealt out to the eight dies in turn: give each a run of tiles that share rows of x and w in its cache.
struct TileAt {
    int m, n;
};
__device__ inline TileAt tile_of(int id, int tiles_m, int tiles_n)
{
    const int all = tiles_m * tiles_n, each = all / kNumXcd, more = all % kNumXcd, die = id % kNumXcd;
    const int t = die * each + min(die, more) + id / kNumXcd;
    const int kBand = 8;              // tiles of a band of rows go down its columns
    const int band = t / (kBand * tiles_n), rows = min(kBand, tiles_m - band * kBand), in = t - band * kBand * tiles_n;
    return {band * kBand + in % rows, in / rows};
}

template <typename T> struct TileType {
    typedef T part_t;
    static const int parts = 1, bk = 64;
};
template <> struct TileType<float> {
    typedef bf16 part_t;
    static const int parts = 3, bk = 32;
};

// fp32 operands are scaled by 2^16 before they are cut into three bf16 numbers, so that the smallest numbers' parts are
// numbers still; what overflows by that shows in the sums, and is summed again as it stands.
static const float kSplitScale = 65536.0f;

// A wave's blocks go to y through LDS, 32 rows at a time, so that y is written (and the residual read) in whole lines.  What
// follows the sums but for the residual stands in the code once, in a loop over LDS; the residual's loads go out before.
// `odd`: the sums are not to be used, they are formed again one by one in fp32.
template <typename T, int TM, int TN>
__device__ inline void put_tile(const LinearArgs &a, const f32x16 (&acc)[TM][TN], float *rows, float scale, bool odd, int slice,
                                int k_begin, int k_end, int m0, int n0)
{
    typedef T tvec __attribute__((ext_vector_type(4)));
    const int kCols = 32 * TN, kPitch = kCols + 4, kQuads = kCols / 4, kStep = 64 / kQuads, kTurns = 32 / kStep;
    const int lane = threadIdx.x & 63, row = lane & 31, half = lane >> 5;
    const int n = n0 + lane % kQuads * 4, n_in = min(n, max(a.n - 4, 0));    // the lane's columns, and ones that there are
    const bool wide = a.wide_y && a.slices == 1, has_n = n < a.n;
    f32x4 bias = {0, 0, 0, 0};
    if (a.bias && wide) bias = __builtin_convertvector(*(const tvec *)((const T *)a.bias + n_in), f32x4);
    float *const mine = rows + lane / kQuads * kPitch + lane % kQuads * 4;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int m = m0 + i * 32 + lane / kQuads;
        tvec res[kTurns];
        if (a.residual && wide)
#pragma unroll
            for (int t = 0; t < kTurns; ++t)
                res[t] = *(const tvec *)((const T *)a.residual + (int64_t)min(m + t * kStep, a.m - 1) * a.residual_stride + n_in);
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *(f32x4 *)&rows[row * kPitch + 32 * j + 2 * r + 4 * half] =
                    f32x4{acc[i][j][r], acc[i][j][r + 1], acc[i][j][r + 2], acc[i][j][r + 3]} * scale;
        if (sizeof(T) == 4 && odd) {
#pragma unroll 1
            for (int e = lane; e < 32 * kCols; e += 64) {
                const T *const xr = (const T *)a.x + (int64_t)min(m0 + i * 32 + e / kCols, a.m - 1) * a.x_stride;
                const T *const wr = (const T *)a.w + (int64_t)min(n0 + e % kCols, a.n - 1) * a.w_stride;
                float sum = 0.0f;
#pragma unroll 1
                for (int k = k_begin; k < k_end; ++k) sum = fmaf((float)xr[k], (float)wr[k], sum);
                rows[e / kCols * kPitch + e % kCols] = sum;
            }
        }
        if (!wide) {
#pragma unroll 1
            for (int t = 0; t < kTurns; ++t)
                finish_or_part<T>(a, slice, m + t * kStep, n, *(const f32x4 *)(mine + t * kStep * kPitch));
            continue;
        }
        if (a.act != WPK_ACT_NONE) {
#pragma unroll 1
            for (int t = 0; t < kTurns; ++t) {
                f32x4 v = *(const f32x4 *)(mine + t * kStep * kPitch) + bias;
                v = a.y_f32 ? apply_act<float>(v, a.act) : apply_act<T>(v, a.act);
                *(f32x4 *)(mine + t * kStep * kPitch) = v;
            }
        }
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
            f32x4 v = *(const f32x4 *)(mine + t * kStep * kPitch);
            if (a.act == WPK_ACT_NONE) v += bias;
            if (a.residual) v += __builtin_convertvector(res[t], f32x4);
            if (!has_n || m + t * kStep >= a.m) continue;
            const int64_t at = (int64_t)(m + t * kStep) * a.y_stride + n;
            if (sizeof(T) == 4 || a.y_f32) *(f32x4 *)((float *)a.y + at) = v;
            else *(tvec *)((T *)a.y + at) = __builtin_convertvector(v, tvec);
        }
    }
}

// BM rows of y (columns of the MFMA) by BN columns, WM x WN waves of 32 x 32 blocks.  A step's operands are held in registers
// while the step before is multiplied, and go to LDS (fp32's cut into their parts on the way) between two meetings of the
// waves.  One LDS buffer: workgroups that share a compute unit fill each other's pauses, which for fp32, whose cutting takes
// two thirds of the products' time, was worth more than a second buffer.  777 x 1000 x 2048 in fp32: 36.3 us with its join (a
// kernel of 4 to 5 us), 88 TFLOP/s, where six bf16 products would take 12 at the rate of large ones: the cutting (six and a half
// vector instructions an element, again by every tile that reads it) has the vector units busy for 36 % of the time, the
// products the matrix pipes for 21 %, and neither fills the other's pauses.
template <typename T, int BM, int BN, int WM, int WN> __global__ void __launch_bounds__(64 * WM * WN) linear_tiles_kernel(LinearArgs a)
{
    typedef typename TileType<T>::part_t part_t;
    typedef typename Mma<part_t>::v8 p8;
    const int NP = TileType<T>::parts, BK = TileType<T>::bk, kRow = BK + 8, kThreads = 64 * WM * WN;
    const int TM = BM / WM / 32, TN = BN / WN / 32, kOctets = BK / 8, kPer = (BM + BN) * kOctets / kThreads;
    static_assert((BM + BN) * kOctets % kThreads == 0 && BN * kOctets % kThreads == 0, "whole rounds of loads");
    const int kPutBytes = 4 * WM * WN * 32 * (32 * TN + 4), kBytes = (BM + BN) * kRow * NP * (int)sizeof(part_t);
    __shared__ __align__(16) unsigned char shared[kBytes > kPutBytes ? kBytes : kPutBytes];
    part_t *const lds = (part_t *)shared;              // [part][rows of w, then rows of x][kRow]
    const int kPart = (BM + BN) * kRow;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = lane & 31, half = lane >> 5;
    const int wm = wave % WM, wn = wave / WM, slice = blockIdx.y;
    const TileAt at = tile_of(blockIdx.x, (a.m + BM - 1) / BM, (a.n + BN - 1) / BN);
    const int m0 = at.m * BM, n0 = at.n * BN;
    const int k_begin = slice * a.slice_k, k_end = min(a.k, k_begin + a.slice_k);

    const T *src[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int task = tid + i * kThreads, r = task / kOctets, o = task % kOctets;
        src[i] = r < BN ? (const T *)a.w + (int64_t)min(n0 + r, a.n - 1) * a.w_stride + 8 * o
                        : (const T *)a.x + (int64_t)min(m0 + r - BN, a.m - 1) * a.x_stride + 8 * o;
    }
    typename Mma<T>::v8 held[kPer];
    auto stage = [&]() {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int task = tid + i * kThreads, to = task / kOctets * kRow + task % kOctets * 8;
            if constexpr (NP == 1) {
                *(p8 *)&lds[to] = held[i];
            } else {
                f32x8 v = held[i] * kSplitScale;
#pragma unroll
                for (int q = 0; q < NP; ++q) {
                    const p8 u = __builtin_convertvector(v, p8);
                    v -= __builtin_convertvector(u, f32x8);
                    *(p8 *)&lds[q * kPart + to] = u;
                }
            }
        }
    };
    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

    auto multiply = [&]() {
#pragma unroll
        for (int s = 0; s < BK / 16; ++s) {
            p8 fw[TN][NP], fx[TM][NP];
#pragma unroll
            for (int q = 0; q < NP; ++q) {
#pragma unroll
                for (int j = 0; j < TN; ++j) fw[j][q] = *(const p8 *)&lds[q * kPart + (wn * TN * 32 + j * 32 + row) * kRow + 16 * s + 8 * half];
#pragma unroll
                for (int i = 0; i < TM; ++i) fx[i][q] = *(const p8 *)&lds[q * kPart + (BN + wm * TM * 32 + i * 32 + row) * kRow + 16 * s + 8 * half];
            }
#pragma unroll
            for (int u = 0; u < NP; ++u)
#pragma unroll
                for (int v = 0; u + v < NP; ++v)
#pragma unroll
                    for (int i = 0; i < TM; ++i)
#pragma unroll
                        for (int j = 0; j < TN; ++j) acc[i][j] = Mma<part_t>::m32(fw[j][u], fx[i][v], acc[i][j]);
        }
    };
    // whole steps, the next one's loads under way without a branch around them (the last whole one's again behind it)
    const int k_whole = k_begin + (k_end - k_begin) / BK * BK;
    if (k_whole > k_begin) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) held[i] = Octet<T>::load(src[i] + k_begin);
        for (int k = k_begin; k < k_whole; k += BK) {
            stage();
            __syncthreads();
            const int next = min(k + BK, k_whole - BK);
#pragma unroll
            for (int i = 0; i < kPer; ++i) held[i] = Octet<T>::load(src[i] + next);
            multiply();
            __syncthreads();
        }
    }
    if (k_whole < k_end) {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            held[i] = Octet<T>::load_some(src[i] + k_whole, k_end - k_whole - (tid + i * kThreads) % kOctets * 8);
        stage();
        __syncthreads();
        multiply();
        __syncthreads();
    }

    float scale = 1.0f;
    bool odd = false;                 // infinities, NaN, or numbers that the scaled parts could not hold
    if constexpr (NP > 1) {
        scale = 1.0f / (kSplitScale * kSplitScale);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) odd = odd || !(fabsf(acc[i][j][r]) <= 3.4028234e38f);
        odd = __any(odd);
    }
    put_tile<T, TM, TN>(a, acc, (float *)shared + wave * 32 * (32 * TN + 4), scale, odd, slice, k_begin, k_end,
                        m0 + wm * TM * 32, n0 + wn * TN * 32);
}

// The same for 16-bit operands in aligned rows: loads write LDS directly and take no registers, STAGES - 1 steps of BK entries
// ahead of the products.  A wave's load brings 1024 bytes of whole rows.  The 16-byte pieces of a row stand in the order of their
// number xor some bits of the row's, which the lanes bring about by what they ask for: 16 lanes that read the same piece of
// neighbouring rows take all banks.  16384 x 4096 x 4096, bf16: 471 us, 1.17 PFLOP/s, the matrix pipes busy 61 % of the time
// (a library product takes 354 to 420); 1777 x 2304 x 1544, f16, GELU: 23.5 us, of which 0.65 a step of 64.  What bounds a step is
// not known: matrix pipes 22 %, vector units 23 % busy, waves waiting for 27 % of their time; the 32 KiB of a step come at 21
// bytes a clock a compute unit, 87 % of the requests met by the L2 caches, 340 clocks each.  (Waves of 64 x 64, two to a block, that read a third
// less of LDS took as long.)
template <typename T, int BM, int BN, int WM, int WN, int BK, int STAGES>
__global__ void __launch_bounds__(64 * WM * WN, (BM + BN) * BK * STAGES * 2 > 81920 ? WM * WN / 4 : WM * WN / 2)
linear_direct_kernel(LinearArgs a)
{
    typedef typename Mma<T>::v8 v8;
    const int kWaves = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    const int kPieces = BK / 8, kLoadRows = 64 / kPieces, kLoads = (BM + BN) / kLoadRows / kWaves;
    static_assert(BN / kLoadRows % kLoads == 0, "a wave loads rows of one matrix");
    __shared__ __align__(16) T lds[STAGES][(BM + BN) * BK];    // rows of w, then rows of x
    static_assert(sizeof(lds) >= sizeof(float) * WM * WN * 32 * (32 * TN + 4), "what put_tile needs");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = lane & 31, half = lane >> 5;
    const int wm = wave % WM, wn = wave / WM, slice = blockIdx.y;
    const TileAt at = tile_of(blockIdx.x, (a.m + BM - 1) / BM, (a.n + BN - 1) / BN);
    const int m0 = at.m * BM, n0 = at.n * BN;
    const int k_begin = slice * a.slice_k, k_end = min(a.k, k_begin + a.slice_k);
    auto order = [](int r) { return BK == 64 ? (r >> 1) & 7 : (r >> 2) & 3; };

    const int w_loads = BN / kLoadRows, load_row = lane / kPieces;
    const bool of_w = wave * kLoads < w_loads;
    const int r0 = (of_w ? n0 : m0) + (wave * kLoads - (of_w ? 0 : w_loads)) * kLoadRows, last = (of_w ? a.n : a.m) - 1;
    const int64_t stride = of_w ? a.w_stride : a.x_stride;
    const int base = min(r0, last);
    const Rows src = __builtin_amdgcn_make_buffer_rsrc((T *)(of_w ? a.w : a.x) + base * stride, 0, 0x7fffffff, 0x00020000);
    auto piece = [&](int i) { return (lane % kPieces ^ order(kLoadRows * (i & 1) + load_row)) * 8; };
    uint32_t from[kLoads];                                     // rows beyond the matrix are read as its last one
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
        from[i] = (uint32_t)((min(r0 + kLoadRows * i + load_row, last) - base) * (int)stride + piece(i)) * sizeof(T);
    const uint32_t lds0 = lds_offset(&lds[0][0]) + wave * kLoads * 1024;
    auto fetch = [&](int stage, int k, int first, int end) {
        const uint32_t to = lds0 + stage * (uint32_t)sizeof(lds[0]);
        const bool whole = k + BK <= k_end;
#pragma unroll
        for (int i = first; i < end; ++i) {
            const uint32_t off = whole || k + piece(i) < k_end ? from[i] : kOutside;      // (outside: zeros)
            load_to_lds(src, off, k * (uint32_t)sizeof(T), to + i * 1024);
        }
    };
    uint32_t read[BK / 16];                                    // where this lane's piece of a block's 16 entries is
#pragma unroll
    for (int s = 0; s < BK / 16; ++s) read[s] = row * BK + ((2 * s + half) ^ order(row)) * 8;

    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

    // A step's blocks of 16 entries are read one ahead of the products, the first of a step with the last products of the step
    // before: between them all waves meet, the step's operands there and the buffer before it read by everyone.  The loads of
    // the step STAGES later go out into that buffer, a share then and the rest behind the reads of the next step's first
    // blocks: all at once they keep the reads waiting (16384 x 4096 x 4096: 502 us against 485).  Steps behind the last
    // are asked for as well, all of them outside, so that the same number of loads is always under way.
    const int kBlocks = BK / 16;
    static_assert(kBlocks % 2 == 0, "blocks alternate between two sets of registers");
    const int kLate = STAGES > 2 ? 2 : 1, kShare = kLoads / (kLate + 1);
    v8 fw[2][TN], fx[2][TM];
    auto read_block = [&](int stage, int s) {
        const T *const pw = &lds[stage][wn * TN * 32 * BK], *const px = &lds[stage][(BN + wm * TM * 32) * BK];
#pragma unroll
        for (int j = 0; j < TN; ++j) fw[s & 1][j] = *(const v8 *)(pw + read[s] + j * 32 * BK);
#pragma unroll
        for (int i = 0; i < TM; ++i) fx[s & 1][i] = *(const v8 *)(px + read[s] + i * 32 * BK);
    };
    auto multiply = [&](int s) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = Mma<T>::m32(fw[s & 1][j], fx[s & 1][i], acc[i][j]);
    };
#pragma unroll
    for (int s = 0; s < STAGES; ++s) fetch(s, k_begin + s * BK, 0, s + 1 < STAGES ? kLoads : kShare);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STAGES - 2) * kLoads + kShare) : "memory");
    __builtin_amdgcn_s_barrier();
    read_block(0, 0);
    int stage = 0;
    for (int k = k_begin; k < k_end; k += BK) {
        const int next = stage == STAGES - 1 ? 0 : stage + 1;
#pragma unroll
        for (int s = 0; s < kBlocks; ++s) {
            if (s + 1 < kBlocks) {
                read_block(stage, s + 1);
            } else {
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((STAGES - 2) * kLoads) : "memory");
                __builtin_amdgcn_s_barrier();
                read_block(next, 0);
            }
            if (s + 1 == kBlocks) fetch(stage, k + STAGES * BK, 0, kShare);
            else if (s < kLate)
                fetch(stage == 0 ? STAGES - 1 : stage - 1, k + (STAGES - 1) * BK, (s + 1) * kShare, s + 1 == kLate ? kLoads : (s + 2) * kShare);
            multiply(s);
            __builtin_amdgcn_sched_barrier(0);
        }
        stage = next;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // (the loads of zeros write LDS too)
    __syncthreads();
    put_tile<T, TM, TN>(a, acc, (float *)&lds[0][0] + wave * 32 * (32 * TN + 4), 1.0f, false, slice, k_begin, k_end,
                        m0 + wm * TM * 32, n0 + wn * TN * 32);
}

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
                    s.slices, s.slice_k, s.width, wide, d.x_stride, d.w_stride, d.y_stride, d.residual_stride, part_stride(d)};
    // (loads that write LDS move 16 aligned bytes)
    const bool direct = d.k % 8 == 0 && d.x_stride % 8 == 0 && d.w_stride % 8 == 0 && aligned_to(x, 16) && aligned_to(w, 16);
    const hipStream_t st = (hipStream_t)stream;
    if (d.dtype == WPK_BF16) return linear_typed<bf16>(a, s, direct, st);
    if (d.dtype == WPK_F16) return linear_typed<f16>(a, s, direct, st);
    return linear_typed<float>(a, s, direct, st);
}

}  // extern "C"
