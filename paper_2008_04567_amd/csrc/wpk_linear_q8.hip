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

// 4 bytes a lane from `rows` at the lane's `offset` plus `step` straight to LDS, as load_to_lds does with 16.
__device__ inline void load_word_to_lds(Rows rows, uint32_t offset, uint32_t step, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n s_nop 0\n buffer_load_dword %0, %1, %3 offen lds"
                 :
                 : "v"(offset), "s"(rows), "s"(lds), "s"(step)
                 : "m0", "memory");
}

typedef const __attribute__((address_space(4))) float *Constants;     // read by scalar loads

// BM rows of y by BN rows of w, WM x WN waves.  Rows go to LDS directly, STAGES - 1 steps ahead, their 16-byte pieces in the
// order of their number xor bits of the row's, so that 16 rows' same pieces take all banks.  The scales of x go there too, eight
// steps' at a time: a load a wave and step brings eight rows' for eight steps, the next eight steps' again and again until these
// begin, so that the same number of loads is always under way.
template <typename T, int BM, int BN, int WM, int WN, int STAGES, bool GROUPED, bool GATED>
__global__ void __launch_bounds__(64 * WM * WN, (BM + BN) * 128 * STAGES > 73728 ? WM * WN / 4 : WM * WN / 2) linear_q8_kernel(Q8Args q)
{
    typedef typename OperandFor<T>::type Operand;
    LinearArgs &a = q.a;
    const int kWaves = WM * WN, BK = 128, TM = BM / WM / 16, TN = BN / WN / 16, kOut = GATED ? BN / 2 : BN;
    const int kPieces = 8, kLoadRows = 8, kLoads = (BM + BN) / kLoadRows / kWaves, kScaleLoads = BM / 8 / kWaves;
    static_assert(BN / kLoadRows % kLoads == 0 && TM % 2 == 0 && TN % 2 == 0 && TM >= 4, "whole loads and blocks");
    static_assert(BM % (8 * kWaves) == 0 && (kScaleLoads & (kScaleLoads - 1)) == 0 && kScaleLoads + STAGES <= 8, "whole loads of scales");
    __shared__ __align__(16) uint8_t lds[STAGES][(BM + BN) * BK];    // rows of w, then rows of x
    __shared__ __align__(16) float scales[2][BM][8];
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
    auto fetch = [&](int stage, int k, int first, int end) {
        const uint32_t to = lds0 + stage * (uint32_t)sizeof(lds[0]);
        const bool whole = k + BK <= k_end;
#pragma unroll
        for (int i = first; i < end; ++i) load_to_lds(src, whole || k + piece(i) < k_end ? from[i] : kOutside, k, to + i * 1024);
    };

    // x's scales: this wave's rows, eight at a time, a step a lane
    const int kb_begin = k_begin / BK, kb_end = (k_end + BK - 1) / BK;
    const bool scales_far = GROUPED && a.source;
    const Rows scale_src = __builtin_amdgcn_make_buffer_rsrc((float *)q.x_scales + (scales_far ? 0 : m0 * q.x_scale_stride), 0, 0x7fffffff, 0x00020000);
    uint32_t scale_from[kScaleLoads];
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
        const int r = x_row<GROUPED>(a, m0 + (wave * kScaleLoads + i) * 8 + lane / 8) - (scales_far ? 0 : m0);
        scale_from[i] = (uint32_t)r * (uint32_t)q.x_scale_stride * 4u + lane % 8 * 4;
    }
    const uint32_t scales0 = lds_offset(&scales[0][0][0]) + wave * kScaleLoads * 256;
    auto fetch_scales = [&](int run, int i) {                  // the i-th load of the steps 8 run .. 8 run + 7
        uint32_t off = scale_from[0];
#pragma unroll
        for (int j = 1; j < kScaleLoads; ++j) off = i == j ? scale_from[j] : off;
        const int kb = kb_begin + 8 * run;
        load_word_to_lds(scale_src, kb + lane % 8 < kb_end ? off : kOutside, kb * 4, scales0 + (run & 1) * (uint32_t)sizeof(scales[0]) + i * 256);
    };
    // (a wave's columns are of one block, or of one in each half)
    const int block = min((n0 + wn * TN * (GATED ? 8 : 16)) / kScaleBlock, (a.n - 1) / kScaleBlock);
    const Constants ws = (Constants)(q.w_scales + (int64_t)block * q.w_scale_stride);
    const Constants ws_up = (Constants)(q.w_scales + (int64_t)(block + (a.n + kScaleBlock - 1) / kScaleBlock) * q.w_scale_stride);

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

    // What is behind a row's end in its last piece is not the row's.
    auto clear_tail = [&](uint8_t *buf, int k) {
        for (int r = tid; r < BM + BN; r += 64 * kWaves) {
            u32x4 *const v = (u32x4 *)(buf + r * BK + (((k_end - k) / 16 ^ order(r)) * 16));
            u32x4 u = *v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int left = min(max((k_end - k) % 16 - 4 * i, 0), 4);
                u[i] &= left == 4 ? 0xffffffffu : (1u << (8 * left)) - 1;
            }
            *v = u;
        }
        __syncthreads();
    };
    const int odd_k = k_end % 16 != 0 ? (k_end - k_begin) / BK * BK + k_begin : -1;      // the step that ends within a piece

    uint32_t at_lo = row * BK + ((2 * g) ^ order(row)) * 16, at_hi = row * BK + ((2 * g + 1) ^ order(row)) * 16;
    auto read = [&](const uint8_t *buf, int r) {               // row r + lane % 16 of a tile (r a multiple of 16), this lane's 32 entries
        const i32x4 lo = *(const i32x4 *)(buf + r * BK + at_lo), hi = *(const i32x4 *)(buf + r * BK + at_hi);
        return (i32x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    const int w_at = wn * TN * 16, x_at = BN + wm * TM * 16;

    // A step's rows of x are read two ahead of the products, the first two and w's with the last products of the step before:
    // between them all waves meet, the step's operands there and the buffer before it read by everyone.
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) fetch_scales(0, i);
#pragma unroll
    for (int s = 0; s < STAGES; ++s) {
        if (s > 0) fetch_scales(0, 0);                         // (again, for the count)
        fetch(s, k_begin + s * BK, 0, kLoads);
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STAGES - 1) * (kLoads + 1)) : "memory");
    __builtin_amdgcn_s_barrier();
    if (odd_k == k_begin) clear_tail(&lds[0][0], k_begin);
    i32x8 fw[TN], fx[2];
#pragma unroll
    for (int j = 0; j < TN; ++j) fw[j] = read(&lds[0][0], w_at + 16 * j);
    fx[0] = read(&lds[0][0], x_at);
    fx[1] = read(&lds[0][0], x_at + 16);
    int stage = 0, step = 0;
    for (int k = k_begin; k < k_end; k += BK, ++step) {
        const int next = stage == STAGES - 1 ? 0 : stage + 1;
        const uint8_t *const buf = &lds[stage][0];
        uint8_t *const buf_next = &lds[next][0];
        const int kb = k / BK;
        const float sw = ws[kb], su = GATED ? ws_up[kb] : sw;
        float sx[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) sx[i] = scales[step >> 3 & 1][wm * TM * 16 + i * 16 + row][step & 7];
        f32x4 v[TN];
        auto add = [&](int i, int j) {
            const float s = sx[i] * (GATED && j % 2 ? su : sw);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][j][r] = fmaf(v[j][r], s, acc[i][j][r]);
            asm volatile("" : "+v"(acc[i][j]));                // (left to itself the compiler adds behind the branch below)
        };
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            if (i == TM - 2) {
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((STAGES - 2) * (kLoads + 1)) : "memory");
                __builtin_amdgcn_s_barrier();
                if (k + BK == odd_k) clear_tail(buf_next, k + BK);
                fetch_scales((step >> 3) + 1, step & (kScaleLoads - 1));
                fetch(stage, k + STAGES * BK, 0, kLoads);
            }
            const Operand x = Operand::of(fx[i & 1]);
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                if (i > 0) add(i - 1, j);
                v[j] = Operand::multiply(Operand::of(fw[j]), x);
                if (i == TM - 1) fw[j] = read(buf_next, w_at + 16 * j);
            }
            fx[i & 1] = i < TM - 2 ? read(buf, x_at + 16 * (i + 2)) : read(buf_next, x_at + 16 * (i + 2 - TM));
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) add(TM - 1, j);
        stage = next;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");     // (the loads of zeros write LDS too)
    __syncthreads();
    float *const rows = (float *)&lds[0][0] + wave * 32 * (16 * TN + 4);
    put_tile<T, TM / 2, TN / 2, GROUPED, GATED>(a, StageSmall<TM, TN>{acc, rows}, rows, false, slice, k_begin, k_end, m0 + wm * TM * 16,
                                                n0 + wn * TN * (GATED ? 8 : 16));
}

template <typename T, int B, int STAGES, bool GROUPED, bool GATED> static int launch_q8(const Q8Args &q, int64_t tiles, hipStream_t st)
{
    if (tiles * 512 >= 1ll << 32) return WPK_E_UNSUPPORTED;
    hipLaunchKernelGGL((linear_q8_kernel<T, B, B, 2, 4, STAGES, GROUPED, GATED>), dim3((unsigned)tiles, q.a.slices), dim3(512), 0, st, q);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

template <typename T> static int linear_q8_typed(const Q8Args &q, hipStream_t st)
{
    auto tiles = [&](int64_t t) { return ((q.a.m + t - 1) / t) * ((q.a.n + t - 1) / t); };
    if constexpr (sizeof(T) == 2)
        if (tiles(256) >= kComputeUnits) return launch_q8<T, 256, 2, false, false>(q, tiles(256), st);
    return launch_q8<T, 128, 4, false, false>(q, tiles(128), st);
}

template <typename T, bool GATED> static int grouped_q8_typed(const Q8Args &q, hipStream_t st)
{
    if constexpr (sizeof(T) == 2)
        if (q.a.m / q.a.groups >= 256) return launch_q8<T, 256, 2, true, GATED>(q, GroupedGrid(q.a, 256, GATED ? 128 : 256).tiles, st);
    return launch_q8<T, 128, 4, true, GATED>(q, GroupedGrid(q.a, 128, GATED ? 64 : 128).tiles, st);
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
