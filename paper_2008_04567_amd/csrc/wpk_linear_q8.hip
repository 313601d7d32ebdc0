// Matrix products of 8-bit operands (e4m3) with a scale for each 128 values of a row of x and each 128 x 128 block of w, plain
// and by expert.
//
// A step of the reduction is 128 entries, a block of scales: its product is formed by matrix instructions from zero, multiplied by
// the row's scale times the weight's, and added to the sums in 32 bits.  As in wpk_product.h, w's rows are the MFMA's rows and x's
// its columns, so a lane's values have one scale of x.
#include "wpk_grouped.h"

namespace wpk {

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// Eight e4m3 numbers as bf16, which holds them exactly.
__device__ inline bf16x8 widen(int32_t lo, int32_t hi)
{
    typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The product of 16 x 16 by 128 entries: lane l holds 32 entries of row l % 16 of either operand.  (Which 32 does not matter as
// long as both operands have them alike.)
// The matrix instruction for 8 bits adds the products of eight neighbouring entries of a lane with 13 bits below the largest of
// them (measured: beside 2^16, 2^3 is kept and 2^2 is not; of different eights everything is), so a sum is off by 1.6e-5 of
// itself where entries are normal: a twentieth of an f16 y's own rounding.  For a y of 32 bits the operands are widened to bf16,
// whose products are added in 32 bits, at half the rate.
struct Operand8 {
    i32x8 v;
    __device__ static Operand8 of(i32x8 v) { return {v}; }
    static __device__ f32x4 multiply(const Operand8 &a, const Operand8 &b)
    {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, f32x4{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
    }
};
struct Operand16 {
    bf16x8 v[4];
    __device__ static Operand16 of(i32x8 v) { return {{widen(v[0], v[1]), widen(v[2], v[3]), widen(v[4], v[5]), widen(v[6], v[7])}}; }
    static __device__ f32x4 multiply(const Operand16 &a, const Operand16 &b)
    {
        f32x4 c = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[i], b.v[i], c, 0, 0, 0);
        return c;
    }
};
template <typename T> struct OperandFor { typedef Operand8 type; };
template <> struct OperandFor<float> { typedef Operand16 type; };

// the sums of blocks of 16 x 16, where a lane holds row l % 16's columns 4 (l / 16) ..
template <int TM, int TN> struct StageSmall {
    const f32x4 (&acc)[TM][TN];
    float *rows;
    __device__ void operator()(int i, int pitch) const
    {
        const int row = threadIdx.x & 15, g = threadIdx.x >> 4 & 3;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < TN; ++j) *(f32x4 *)&rows[(16 * h + row) * pitch + 16 * j + 4 * g] = acc[2 * i + h][j];
    }
};

// BM rows of y by BN rows of w, WM x WN waves.  Rows go to LDS directly, STAGES - 1 steps ahead, their 16-byte pieces in the
// order of their number xor bits of the row's, so that 16 rows' same pieces take all banks.
template <typename T, int BM, int BN, int WM, int WN, int STAGES, bool GROUPED, bool GATED>
__global__ void __launch_bounds__(64 * WM * WN) linear_q8_kernel(Q8Args q)
{
    typedef typename OperandFor<T>::type Operand;
    LinearArgs &a = q.a;
    const int kWaves = WM * WN, BK = 128, TM = BM / WM / 16, TN = BN / WN / 16, kOut = GATED ? BN / 2 : BN;
    const int kPieces = 8, kLoadRows = 8, kLoads = (BM + BN) / kLoadRows / kWaves;
    static_assert(BN / kLoadRows % kLoads == 0 && TM % 2 == 0 && TN % 2 == 0, "whole loads and blocks");
    __shared__ __align__(16) uint8_t lds[STAGES][(BM + BN) * BK];    // rows of w, then rows of x
    static_assert(sizeof(lds) >= sizeof(float) * WM * WN * 32 * (16 * TN + 4), "what put_tile needs");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = lane & 15, g = lane >> 4;
    const int wm = wave % WM, wn = wave / WM, slice = GROUPED ? 0 : blockIdx.y;
    TileAt at = {0, 0};
    if constexpr (GROUPED) {
        GroupTile tile;
        if (!take_group_tile<BM>(a, blockIdx.x, (a.n + kOut - 1) / kOut, 1, sizeof(T), &tile)) return;
        at.n = tile.n;
        q.w_scales += tile.group * q.w_scale_group_stride;
        if (!a.source) q.x_scales += tile.row * q.x_scale_stride;
    } else {
        at = tile_of(blockIdx.x, (a.m + BM - 1) / BM, (a.n + BN - 1) / BN);
    }
    const int m0 = at.m * BM, n0 = at.n * kOut;
    const int k_begin = slice * a.slice_k, k_end = min(a.k, k_begin + a.slice_k);
    auto order = [](int r) { return (r >> 1) & 7; };

    const int w_loads = BN / kLoadRows, load_row = lane / kPieces;
    const bool of_w = wave * kLoads < w_loads;
    const int in_tile = (wave * kLoads - (of_w ? 0 : w_loads)) * kLoadRows;
    const int r0 = (of_w ? n0 : m0) + in_tile, last = (of_w ? a.n : a.m) - 1;
    const int64_t stride = of_w ? a.w_stride : a.x_stride;
    const bool far = of_w ? GATED : GROUPED && a.source;
    const int base = far ? 0 : min(r0, last);
    const Rows src = __builtin_amdgcn_make_buffer_rsrc((uint8_t *)(of_w ? a.w : a.x) + base * stride, 0, 0x7fffffff, 0x00020000);
    auto piece = [&](int i) { return (lane % kPieces ^ order(kLoadRows * (i & 1) + load_row)) * 16; };
    uint32_t from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int r = kLoadRows * i + load_row;
        const int row_at = !far ? min(r0 + r, last) : of_w ? w_row<GATED>(a, n0, in_tile + r) : x_row<GROUPED>(a, r0 + r);
        from[i] = (uint32_t)(row_at - base) * (uint32_t)stride + piece(i);
    }
    const uint32_t lds0 = lds_offset(&lds[0][0]) + wave * kLoads * 1024;
    auto fetch = [&](int stage, int k) {
        const uint32_t to = lds0 + stage * (uint32_t)sizeof(lds[0]);
        const bool whole = k + BK <= k_end;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load_to_lds(src, whole || k + piece(i) < k_end ? from[i] : kOutside, k, to + i * 1024);
    };

    const float *xs[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) xs[i] = q.x_scales + (int64_t)x_row<GROUPED>(a, m0 + (wm * TM + i) * 16 + row) * q.x_scale_stride;
    // (a wave's columns are of one block, or of one in each half)
    const int block = (n0 + wn * TN * (GATED ? 8 : 16)) / kScaleBlock;
    const float *const ws = q.w_scales + (int64_t)min(block, (a.n - 1) / kScaleBlock) * q.w_scale_stride;
    const float *const ws_up = ws + (int64_t)((a.n + kScaleBlock - 1) / kScaleBlock) * q.w_scale_stride;

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) fetch(s, k_begin + s * BK);
    int stage = 0;
    for (int k = k_begin; k < k_end; k += BK) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((STAGES - 2) * kLoads) : "memory");
        __builtin_amdgcn_s_barrier();
        fetch(stage == 0 ? STAGES - 1 : stage - 1, k + (STAGES - 1) * BK);
        uint8_t *const buf = &lds[stage][0];
        if (k + BK > k_end && k_end % 16 != 0) {               // what is behind a row's end in its last piece is not the row's
            for (int r = tid; r < BM + BN; r += 64 * kWaves) {
                const int p = (k_end - k) / 16;
                u32x4 *const v = (u32x4 *)(buf + r * BK + ((p ^ order(r)) * 16));
                u32x4 u = *v;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int left = min(max((k_end - k) % 16 - 4 * i, 0), 4);
                    u[i] &= left == 4 ? 0xffffffffu : (1u << (8 * left)) - 1;
                }
                *v = u;
            }
            __syncthreads();
        }
        auto read = [&](int r) {                               // row r of the tile, this lane's 32 entries
            const uint8_t *const p = buf + r * BK;
            const i32x4 lo = *(const i32x4 *)(p + ((2 * g) ^ order(r)) * 16), hi = *(const i32x4 *)(p + ((2 * g + 1) ^ order(r)) * 16);
            return Operand::of(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        const int kb = k / BK;
        float sx[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) sx[i] = xs[i][kb];
        const float sw = ws[kb], su = GATED ? ws_up[kb] : sw;
        Operand fw[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) fw[j] = read(wn * TN * 16 + j * 16 + row);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const Operand fx = read(BN + (wm * TM + i) * 16 + row);
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const f32x4 v = Operand::multiply(fw[j], fx);
                const float s = sx[i] * (GATED && j % 2 ? su : sw);
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][j][r] = fmaf(v[r], s, acc[i][j][r]);
            }
        }
        stage = stage == STAGES - 1 ? 0 : stage + 1;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // (the loads of zeros write LDS too)
    __syncthreads();
    float *const rows = (float *)&lds[0][0] + wave * 32 * (16 * TN + 4);
    put_tile<T, TM / 2, TN / 2, GROUPED, GATED>(a, StageSmall<TM, TN>{acc, rows}, rows, false, slice, k_begin, k_end, m0 + wm * TM * 16,
                                                n0 + wn * TN * (GATED ? 8 : 16));
}

template <typename T> static int linear_q8_typed(const Q8Args &q, hipStream_t st)
{
    const LinearArgs &a = q.a;
    const int64_t tiles = (int64_t)((a.m + 127) / 128) * ((a.n + 127) / 128);
    if (tiles * 512 >= 1ll << 32) return WPK_E_UNSUPPORTED;
    hipLaunchKernelGGL((linear_q8_kernel<T, 128, 128, 2, 4, 4, false, false>), dim3((unsigned)tiles, a.slices), dim3(512), 0, st, q);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

template <typename T, bool GATED> static int grouped_q8_typed(const Q8Args &q, hipStream_t st)
{
    const GroupedGrid g(q.a, 128, GATED ? 64 : 128);
    if (g.too_large(512)) return WPK_E_UNSUPPORTED;
    hipLaunchKernelGGL((linear_q8_kernel<T, 128, 128, 2, 4, 4, true, GATED>), dim3(g.all), dim3(512), 0, st, q);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

int grouped_q8(const Q8Args &q, int y_dtype, bool gated, hipStream_t st)
{
    // Loads reach 2^31 bytes from the first row where rows are looked up or a weight has two halves.
    const int64_t far = 1ll << 31;
    if ((q.a.source && q.a.x_rows * q.a.x_stride >= far) || (gated && 2ll * q.a.n * q.a.w_stride >= far)) return WPK_E_UNSUPPORTED;
    if (y_dtype == WPK_BF16) return gated ? grouped_q8_typed<bf16, true>(q, st) : grouped_q8_typed<bf16, false>(q, st);
    if (y_dtype == WPK_F16) return gated ? grouped_q8_typed<f16, true>(q, st) : grouped_q8_typed<f16, false>(q, st);
    return gated ? grouped_q8_typed<float, true>(q, st) : grouped_q8_typed<float, false>(q, st);
}

static int check_linear_q8(const wpk_linear_q8_desc *dp)
{
    if (!dp) return WPK_E_NULL_PTR;
    const wpk_linear_q8_desc &d = *dp;
    if (d.m < 0 || d.n < 1 || d.k < 1 || d.x_stride < d.k || d.w_stride < d.k || d.y_stride < d.n || d.residual_stride < d.n ||
        d.x_scale_stride < scale_blocks(d.k) || d.w_scale_stride < scale_blocks(d.k))
        return WPK_E_BAD_DESC;
    const int64_t most = 1ll << 20;
    if (d.m > kMostRows || d.n > kMostRows || !seq_type_ok(d.dtype) || d.act < WPK_ACT_NONE || d.act > WPK_ACT_GELU || d.reserved != 0 ||
        d.x_stride >= most || d.w_stride >= most || d.y_stride >= most || d.residual_stride >= most || d.x_scale_stride >= most ||
        d.w_scale_stride >= most || d.x_stride % 16 != 0 || d.w_stride % 16 != 0)
        return WPK_E_UNSUPPORTED;
    return WPK_OK;
}

}  // namespace wpk

extern "C" {

int64_t wpk_linear_q8_workspace_bytes(const wpk_linear_q8_desc *d)
{
    return wpk::check_linear_q8(d);
}

int wpk_linear_q8_fwd(const wpk_linear_q8_desc *dp, const void *x, const float *x_scales, const void *w, const float *w_scales,
                      const void *bias, const void *residual, void *y, void *workspace, void *stream)
{
    using namespace wpk;
    const int rc = check_linear_q8(dp);
    if (rc != WPK_OK) return rc;
    const wpk_linear_q8_desc d = *dp;
    if (d.m == 0) return WPK_OK;
    if (!x || !x_scales || !w || !w_scales || !y) return WPK_E_NULL_PTR;
    const size_t e = seq_type_bytes(d.dtype);
    if (!aligned_to(x, 16) || !aligned_to(w, 16) || !aligned_to(x_scales, 4) || !aligned_to(w_scales, 4) || !aligned_to(bias, e) ||
        !aligned_to(residual, e) || !aligned_to(y, e) || !aligned_to(workspace, 16))
        return WPK_E_BAD_ARG;
    const bool wide = d.n % 4 == 0 && d.y_stride % 4 == 0 && aligned_to(y, 4 * e) && aligned_to(bias, 4 * e) &&
                      (!residual || (d.residual_stride % 4 == 0 && aligned_to(residual, 4 * e)));
    const LinearArgs a = {x, w, bias, residual, y, (float *)workspace, d.m, d.n, d.k, d.act, d.dtype == WPK_F32, 1, (d.k + 127) / 128 * 128,
                          64, wide, d.x_stride, d.w_stride, d.y_stride, d.residual_stride, ((int64_t)d.n + 3) / 4 * 4, nullptr, nullptr,
                          1, d.m, 0};
    const Q8Args q = {a, x_scales, w_scales, d.x_scale_stride, d.w_scale_stride, 0};
    const hipStream_t st = (hipStream_t)stream;
    if (d.dtype == WPK_BF16) return linear_q8_typed<bf16>(q, st);
    if (d.dtype == WPK_F16) return linear_q8_typed<f16>(q, st);
    return linear_q8_typed<float>(q, st);
}

}  // extern "C"
