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
// them (measured: beside 2^16, 2^3 is kept and 2^2 is not, also where a -2^16 takes the 2^16 away; of different eights everything that
// 32 bits hold is; the instruction for 32 entries does the same).  Seven of an eight lose up to 2^-13 of the largest each: a sum is off
// by 7 2^-13 of the eights' largest magnitudes at most, by 1.6e-5 of itself where entries are normal, by some 1e-4 where every
// eight has one product of 2^15 beside such of 2^1, and by half where two of 2^15 cancel in every eight.  Values of 8 bits are off by up
// to 2^-4 themselves, so a y of 16 bits takes that for twice the rate.  For a y of 32 bits the operands are widened to bf16, whose
// products are added in 32 bits: 16384 x 4096 x 4096 578 us against 247, 2048 x 4096 x 4096 82 against 54, 32 x 8512 x 2048 7.7 either
// way.  (In tiles of 256 and 128 the widened operands would not fit the registers.)
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

// BM rows of y by BN rows of w, WM x WN waves.  Rows go to LDS directly, their 16-byte pieces in the order of their number xor bits
// of the row's, so that reads meet no bank twice.  The waves meet twice a step: the first time w's rows and the first half of a
// wave's rows of x have been read by everyone and go to the step STAGES later, the second time the rest; so every load has a step
// and a half of two steps' room to arrive.  The scales of x go to LDS too, eight steps' at a time: a load a wave and step brings
// eight rows' for eight steps, the next eight steps' again and again until these begin, so that the same number of loads is always
// under way.  (Every other eight rows have the two halves of the eight steps exchanged, so that 16 rows' scales of a step take 16
// banks.)
// In the form of 64 rows this is not so: a wave has two loads of scales there, and the compiler keeps the choice between their offsets in
// scratch memory (12 bytes a lane) and waits for every load under way when it reads it, once a step.  Its steps therefore last as
// long as their loads do, and its times below are of that.
// 16384 x 4096 x 4096, bf16: 255 us, 274 to 285 with a residual, 1.93 PFLOP/s and more (a library product with one scale for all
// takes 192 and no residual).  A step of 256 x 256 takes 1.7 us on a full device where its products alone take 1.04 (the matrix pipes are
// busy 44 % of the cycles), 1.3 on one workgroup alone.  Without its loads it takes 1.4, without the multiplications by scales 1.4,
// and fewer cycles came with lower clocks (2.28 to 2.12 GHz): the steps are bound by power more than by any unit.  52 us of the
// whole, 73 with a residual, are beginnings and ends of tiles (from times at reductions of 128 and more): a compute unit has room for
// one workgroup, so it is idle while a tile's first steps arrive, and all of them write at once.  Tried without gain: one meeting a step, four steps in LDS (one workgroup a compute unit instead of three: 24 against
// 13.5 us for 65 x 8512 x 2048), waves of 64 x 64 in tiles of 128, tiles of 128 x 256, a tile's residual asked for a block ahead.
template <typename T, int BM, int BN, int WM, int WN, int STAGES, bool GROUPED, bool GATED>
__global__ void __launch_bounds__(64 * WM * WN, (BM + BN) * 128 * STAGES > 73728 ? WM * WN / 4 : WM * WN / 2) linear_q8_kernel(Q8Args q)
{
    typedef typename OperandFor<T>::type Operand;
    LinearArgs &a = q.a;
    const int kWaves = WM * WN, BK = 128, TM = BM / WM / 16, TN = BN / WN / 16, kOut = GATED ? BN / 2 : BN;
    const int kWLoads = BN / 8 / kWaves, kXLoads = BM / 16 / kWaves, kLoads = kWLoads + 2 * kXLoads, kScaleLoads = BM / 8 / kWaves;
    static_assert(BN % (8 * kWaves) == 0 && BM % (16 * kWaves) == 0 && TM % 4 == 0 && TN % 2 == 0, "whole loads and blocks");
    static_assert(BM % (8 * kWaves) == 0 && kScaleLoads % 2 == 0 && (kScaleLoads & (kScaleLoads - 1)) == 0 && kScaleLoads + STAGES <= 8, "whole loads of scales");
    __shared__ __align__(16) uint8_t lds[STAGES][(BM + BN) * BK];    // rows of w, then rows of x
    __shared__ __align__(16) float scales[2][BM][8];
    static_assert(sizeof(lds) >= sizeof(float) * WM * WN * 32 * (16 * TN + 4), "what put_tile needs");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = lane & 15, g = lane >> 4;
    // (waves of different rows share a SIMD: where a tile has no rows for one of them, the other has it to itself)
    const int wm = wave / WN, wn = wave % WN, slice = GROUPED ? 0 : blockIdx.y;
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

    // A load brings eight rows' 128 bytes.  A wave's: rows of w, then of the first halves of the waves' rows of x, then of the second.
    // (Rows that are looked up, and both halves of a gated weight, are reached from the matrix' first row.)
    const bool far = GROUPED && a.source;
    const int w_base = GATED ? 0 : n0;
    const Rows w_src = __builtin_amdgcn_make_buffer_rsrc((uint8_t *)a.w + w_base * a.w_stride, 0, 0x7fffffff, 0x00020000);
    const Rows x_src = __builtin_amdgcn_make_buffer_rsrc((uint8_t *)a.x + (far ? 0 : m0 * a.x_stride), 0, 0x7fffffff, 0x00020000);
    auto lds_row = [&](int i) {                                // of the wave's i-th load
        if (i < kWLoads) return (wave * kWLoads + i) * 8;
        const int q = (wave * kXLoads + (i - kWLoads) % kXLoads) * 8, half = (i - kWLoads) / kXLoads;
        return BN + q / (TM * 8) * (TM * 16) + half * TM * 8 + q % (TM * 8);
    };
    auto piece = [&](int i) { return (lane % 8 ^ order((lds_row(i) + lane / 8) % 16)) * 16; };
    uint32_t from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int r = lds_row(i) + lane / 8;
        from[i] = i < kWLoads ? (uint32_t)(w_row<GATED>(a, n0, r) - w_base) * (uint32_t)a.w_stride
                              : (uint32_t)(x_row<GROUPED>(a, m0 + r - BN) - (far ? 0 : m0)) * (uint32_t)a.x_stride;
        from[i] += piece(i);
    }
    const uint32_t lds0 = lds_offset(&lds[0][0]);
    auto fetch = [&](int stage, int k, int first, int end) {
        const uint32_t to = lds0 + stage * (uint32_t)sizeof(lds[0]);
        const bool whole = k + BK <= k_end;
#pragma unroll
        for (int i = first; i < end; ++i)
            load_to_lds(i < kWLoads ? w_src : x_src, whole || k + piece(i) < k_end ? from[i] : kOutside, k, to + lds_row(i) * BK);
    };

    // x's scales: this wave's rows, eight at a time, a step a lane
    const int kb_begin = k_begin / BK, kb_end = (k_end + BK - 1) / BK;
    const Rows scale_src = __builtin_amdgcn_make_buffer_rsrc((float *)q.x_scales + (far ? 0 : m0 * q.x_scale_stride), 0, 0x7fffffff, 0x00020000);
    uint32_t scale_from[kScaleLoads];
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
        const int r = x_row<GROUPED>(a, m0 + (wave * kScaleLoads + i) * 8 + lane / 8) - (far ? 0 : m0);
        scale_from[i] = (uint32_t)r * (uint32_t)q.x_scale_stride * 4u + (lane % 8 ^ 4 * (i & 1)) * 4;
    }
    const uint32_t scales0 = lds_offset(&scales[0][0][0]) + wave * kScaleLoads * 256;
    auto fetch_scales = [&](int run, int i) {                  // the i-th load of the steps 8 run .. 8 run + 7
        uint32_t off = scale_from[0];
#pragma unroll
        for (int j = 1; j < kScaleLoads; ++j) off = i == j ? scale_from[j] : off;
        const int kb = kb_begin + 8 * run;
        load_word_to_lds(scale_src, kb + (lane % 8 ^ 4 * (i & 1)) < kb_end ? off : kOutside, kb * 4, scales0 + (run & 1) * (uint32_t)sizeof(scales[0]) + i * 256);
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

    // What is behind a row's end in its last piece is not the row's.  (half: of x's rows, whose first half comes with w's)
    auto clear_tail = [&](uint8_t *buf, int k, int half) {
        for (int r = tid; r < BM + BN; r += 64 * kWaves) {
            if ((r >= BN && (r - BN) / (TM * 8) % 2 == 1) != (half == 1)) continue;
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

    // (a lane's pieces are g and g + 4: LDS serves lanes 0-3, 12-15 and 20-27 of a read together, and so on, and with 2 g and 2 g + 1
    // two of these would meet in every bank)
    const uint32_t at_lo = row * BK + (g ^ order(row)) * 16, at_hi = at_lo ^ 64;
    auto read = [&](const uint8_t *buf, int r) {               // row r + lane % 16 of a tile (r a multiple of 16), this lane's 32 entries
        const i32x4 lo = *(const i32x4 *)(buf + r * BK + at_lo), hi = *(const i32x4 *)(buf + r * BK + at_hi);
        return (i32x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    const int w_at = wn * TN * 16, x_at = BN + wm * TM * 16;

    // Blocks of x's rows are taken in pairs, all of w's with the one and the other in turn, and read a pair ahead; w's for the next
    // step as soon as the last pair has been multiplied with them.  Sums are added to four products later.
    const int kFirst = kWLoads + kXLoads, kMeet1 = TM / 4 - 1, kMeet2 = TM / 2 - 1, kAhead = 4, kUnderWay = (STAGES - 1) * (kLoads + 1);
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) fetch_scales(0, i);
#pragma unroll
    for (int s = 0; s < STAGES; ++s) {
        fetch(s, k_begin + s * BK, 0, kFirst);
        fetch_scales(0, 0);                                    // (again, for the count)
        fetch(s, k_begin + s * BK, kFirst, kLoads);
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kUnderWay + kXLoads + 1) : "memory");
    __builtin_amdgcn_s_barrier();
    if (odd_k == k_begin) clear_tail(&lds[0][0], k_begin, 0);
    int stage = 0, step = 0;
    if (WM > 1 && m0 + wm * TM * 16 >= a.m) {                  // no rows for this wave: it loads, meets and clears as the others do
        for (int k = k_begin; k < k_end; k += BK, ++step) {
            const int next = stage == STAGES - 1 ? 0 : stage + 1;
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kUnderWay) : "memory");
            __builtin_amdgcn_s_barrier();
            if (k == odd_k) clear_tail(&lds[stage][0], k, 1);
            fetch(stage, k + STAGES * BK, 0, kFirst);
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kUnderWay) : "memory");
            __builtin_amdgcn_s_barrier();
            if (k + BK == odd_k) clear_tail(&lds[next][0], k + BK, 0);
            fetch_scales((step >> 3) + 1, step & (kScaleLoads - 1));
            fetch(stage, k + STAGES * BK, kFirst, kLoads);
            stage = next;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        return;
    }
    i32x8 fw[TN], fx[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) fx[0][h] = read(&lds[0][0], x_at + 16 * h);
#pragma unroll
    for (int j = 0; j < TN; ++j) fw[j] = read(&lds[0][0], w_at + 16 * j);
    for (int k = k_begin; k < k_end; k += BK, ++step) {
        const int next = stage == STAGES - 1 ? 0 : stage + 1;
        uint8_t *const buf = &lds[stage][0], *const buf_next = &lds[next][0];
        const int kb = k / BK;
        const float sw = ws[kb], su = GATED ? ws_up[kb] : sw;
        float sx[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) sx[i] = scales[step >> 3 & 1][wm * TM * 16 + i * 16 + row][(step & 7) ^ (row >> 3 << 2)];
        f32x4 v[kAhead];
        auto add = [&](int p) {                                // the p-th product of the step
            const int i = p / (2 * TN) * 2 + p % 2, j = p / 2 % TN;
            const float s = sx[i] * (GATED && j % 2 ? su : sw);
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][j][r] = fmaf(v[p % kAhead][r], s, acc[i][j][r]);
            asm volatile("" : "+v"(acc[i][j]));                // (left to itself the compiler adds behind the branch below)
        };
#pragma unroll
        for (int i = 0; i < TM / 2; ++i) {
            if (i == kMeet1 || i == kMeet2) {
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kUnderWay) : "memory");
                __builtin_amdgcn_s_barrier();
            }
            if (i == kMeet1 && k == odd_k) clear_tail(buf, k, 1);
            if (i == kMeet2 && k + BK == odd_k) clear_tail(buf_next, k + BK, 0);
            const bool last = i == TM / 2 - 1;
#pragma unroll
            for (int j = 0; j < TN; ++j) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int p = i * 2 * TN + 2 * j + h;
                    if (p >= kAhead) add(p - kAhead);
                    v[p % kAhead] = Operand::multiply(Operand::of(fw[j]), Operand::of(fx[i % 2][h]));
                }
                if (i >= kMeet1 && i < kMeet2) {
                    const int slots = (kMeet2 - kMeet1) * TN, at = (i - kMeet1) * TN + j;
                    fetch(stage, k + STAGES * BK, kFirst * at / slots, kFirst * (at + 1) / slots);
                } else if (i == kMeet2) {
                    if (j == 0) fetch_scales((step >> 3) + 1, step & (kScaleLoads - 1));
                    fetch(stage, k + STAGES * BK, kFirst + kXLoads * j / TN, kFirst + kXLoads * (j + 1) / TN);
                }
                if (j < 2) fx[(i + 1) % 2][j] = last ? read(buf_next, x_at + 16 * j) : read(buf, x_at + 32 * (i + 1) + 16 * j);
                if (last) fw[j] = read(buf_next, w_at + 16 * j);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int p = TM * TN - kAhead; p < TM * TN; ++p) add(p);
        stage = next;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");     // (the loads of zeros write LDS too)
    __syncthreads();
    float *const rows = (float *)&lds[0][0] + wave * 32 * (16 * TN + 4);
    put_tile<T, TM / 2, TN / 2, GROUPED, GATED>(a, StageSmall<TM, TN>{acc, rows}, rows, false, slice, k_begin, k_end, m0 + wm * TM * 16,
                                                n0 + wn * TN * (GATED ? 8 : 16));
}

// ---- few rows ------------------------------------------------------------------------------------------------
// As product_rows: a workgroup of eight waves owns `width` columns of y (of each half, GATED), 16 NT at most together, and all of
// up to 16 MT rows.  A wave takes every eighth block of 128 entries of its slice, U of them under way, w straight into registers.  32
// rows by 8512 columns of 2048: 7.6 us (workgroups of 16 columns 12.8, of 32 11.8, of 36 7.6), of which a launch and one latency are
// most: w's bytes alone take 3.4.  That is with w in the caches; with weights that rotate through 430 MB 8.7, one row 6.4 instead of 5.0.
// (By expert x and w are read by flat instructions, and a wait for one block is a wait for all under way: see `uniform`.)
template <typename T, int MT, int NT, int U, bool GROUPED, bool GATED>
__global__ void __launch_bounds__(64 * kRowsWaves) linear_q8_rows_kernel(Q8Args q)
{
    typedef typename OperandFor<T>::type Operand;
    const int BK = 128;
    LinearArgs &a = q.a;
    __shared__ __align__(16) f32x4 sums[kRowsWaves][MT * NT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 15, g = lane >> 4;
    GroupTile tile = {(int)blockIdx.x, 0, 0};
    if constexpr (GROUPED) {
        if (!take_group_tile<16 * MT>(a, blockIdx.x, (a.n + a.width - 1) / a.width, 1, sizeof(T), &tile)) return;
        q.w_scales += tile.group * q.w_scale_group_stride;
        if (!a.source) q.x_scales += tile.row * q.x_scale_stride;
    }
    const int n0 = tile.n * a.width, n_end = min(n0 + a.width, a.n), slice = GROUPED ? 0 : blockIdx.y;
    const int k_end = min(a.k, (slice + 1) * a.slice_k), k_begin = slice * a.slice_k + BK * wave;
    const uint8_t *wp[NT], *xp[MT];
    const float *ws[NT], *xs[MT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int c = n0 + 16 * (GATED ? i / 2 : i);
        wp[i] = (const uint8_t *)a.w + ((int64_t)min(c + row, n_end - 1) + (GATED ? i % 2 * a.n : 0)) * a.w_stride + 32 * g;
        // (the four columns that a lane has the sums of are of one block)
        const int block = min(c + 4 * g, n_end - 1) / kScaleBlock + (GATED ? i % 2 * ((a.n + kScaleBlock - 1) / kScaleBlock) : 0);
        ws[i] = q.w_scales + (int64_t)block * q.w_scale_stride;
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t r = x_row<GROUPED>(a, 16 * i + row);
        xp[i] = (const uint8_t *)a.x + r * a.x_stride + 32 * g;
        xs[i] = q.x_scales + r * q.x_scale_stride;
    }
    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

    auto load = [](const uint8_t *p) {
        const i32x4 lo = *(const i32x4 *)p, hi = *(const i32x4 *)(p + 16);
        return (i32x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto load_some = [](const uint8_t *p, int left) {          // `left` entries are there
        i32x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (left <= 16 * h) continue;
            const i32x4 u = *(const i32x4 *)(p + 16 * h);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int bytes = min(max(left - 16 * h - 4 * i, 0), 4);
                v[4 * h + i] = bytes == 4 ? u[i] : u[i] & (int32_t)((1u << (8 * bytes)) - 1);
            }
        }
        return v;
    };
    i32x8 fw[U][NT], fx[U][MT];
    float sw[U][NT], sx[U][MT];
    auto fetch_scales = [&](int u, int kb) {
#pragma unroll
        for (int i = 0; i < NT; ++i) sw[u][i] = ws[i][kb];
#pragma unroll
        for (int i = 0; i < MT; ++i) sx[u][i] = xs[i][kb];
    };
    auto fetch = [&](int u, int k) {
#pragma unroll
        for (int i = 0; i < NT; ++i) fw[u][i] = load(wp[i] + k);
#pragma unroll
        for (int i = 0; i < MT; ++i) fx[u][i] = load(xp[i] + k);
        fetch_scales(u, k / BK);
    };
    auto multiply = [&](int u) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const Operand x = Operand::of(fx[u][i]);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const f32x4 v = Operand::multiply(Operand::of(fw[u][j]), x);
                const float s = sx[u][i] * sw[u][j];
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][j][r] = fmaf(v[r], s, acc[i][j][r]);
            }
        }
    };
    const int step = BK * kRowsWaves;
    int k = k_begin;
    if (k + (U - 1) * step + BK <= k_end) {
#pragma unroll
        for (int u = 0; u < U; ++u) fetch(u, k + u * step);
        for (; k + (2 * U - 1) * step + BK <= k_end; k += U * step) {
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
    for (; k + BK <= k_end; k += step) {
        fetch(0, k);
        multiply(0);
    }
    if (k < k_end) {                  // the reduction's last entries, fewer than 128
        const int left = k_end - k - 32 * g;
#pragma unroll
        for (int i = 0; i < NT; ++i) fw[0][i] = load_some(wp[i] + k, left);
#pragma unroll
        for (int i = 0; i < MT; ++i) fx[0][i] = load_some(xp[i] + k, left);
        fetch_scales(0, k / BK);
        multiply(0);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) sums[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    auto sum_of = [&](int t) {
        f32x4 v = sums[0][t][lane];
#pragma unroll
        for (int s = 1; s < kRowsWaves; ++s) v += sums[s][t][lane];
        return v;
    };
    if constexpr (GATED) {
        for (int t = wave; t < MT * NT / 2; t += kRowsWaves) {
            const int n = n0 + 16 * (t % (NT / 2)) + 4 * g;
            const f32x4 v = gate<T>(a, sum_of(2 * t), sum_of(2 * t + 1));
            if (n < n_end) finish<T>(a, 16 * (t / (NT / 2)) + row, n, v, WPK_ACT_NONE);
        }
    } else {
        for (int t = wave; t < MT * NT; t += kRowsWaves) {
            const f32x4 v = sum_of(t);
            const int n = n0 + 16 * (t % NT) + 4 * g;
            if (n < n_end) finish_or_part<T>(a, slice, 16 * (t / NT) + row, n, v);
        }
    }
}

// ---- which of them ----------------------------------------------------------------------------------------------
// Rows of x that the row kernel takes: 64 rows by 8512 columns of 2048 take 11.0 us, 65 (tiles) 13.5.
static const int kQ8RowsMost = 64;
enum { kQ8Rows = 0, kQ8Tile64 = 64, kQ8Tile128 = 128, kQ8Tile256 = 256 };      // rows of a tile (64: by 128 of w)
struct Q8Shape {
    int form, width, slices, slice_k;         // width: as LinearShape's
};

static Q8Shape q8_shape(int64_t m, int64_t n, int64_t k, int dtype)
{
    Q8Shape s = {kQ8Rows, 0, 1, (int)((k + 127) / 128 * 128)};
    const int64_t steps = (k + 127) / 128;
    int64_t slices = 1;
    if (m <= kQ8RowsMost) {
        // (as linear_shape has it; each of the eight waves keeps two blocks of 128 at least)
        const int least = m <= 4 ? 4 : m <= 16 ? 8 : 16;
        const int64_t rounds = (n + 48 * kComputeUnits - 1) / (48 * kComputeUnits);
        const int64_t even = (n + rounds * kComputeUnits - 1) / (rounds * kComputeUnits);
        s.width = (int)((even > least ? even : least) + 3) / 4 * 4;
        slices = kComputeUnits / ((n + s.width - 1) / s.width);
        if (slices > steps / (2 * kRowsWaves)) slices = steps / (2 * kRowsWaves);
    } else {
        // A step of small tiles takes 0.6 us and waits for all loads that are under way (above); three workgroups that share a compute
        // unit hide part of each other's waits; large ones are bound by power and read less.  us, tiles of 64 / 128 / 256, bf16 y:
        //   m x n x k   1024 x 4096 x 4096   2048 x 8512 x 2048   2048 x 4096 x 4096   4096 x 4096 x 1024   16384 x 4096 x 1024
        //               34 / 40 / 48         64 / 63 / 73         63 / 55 / 62         34 / 40 / 36         125 / 109 / 95
        // Sums in bf16 operands (fp32 y) take more registers and time: 2048 x 4096 x 4096 85 / 98.
        const int64_t small = ((m + 63) / 64) * ((n + 127) / 128), large = ((m + 255) / 256) * ((n + 255) / 256);
        const bool wide = dtype != WPK_F32;
        s.form = wide && large >= kComputeUnits && (k > 1024 || large >= 4 * kComputeUnits) ? kQ8Tile256
                 : wide && small > 3 * kComputeUnits && k >= 4096                           ? kQ8Tile128
                                                                                            : kQ8Tile64;
        if (s.form == kQ8Tile64) {
            // (Of tiles that wait for their loads in every step, as all figures here.)
            // The reduction is cut where steps are worth more than another kernel and the partial sums, written and read: 0.6 us a
            // step in turns of all the workgroups that there is room for, 4 us, and 8 bytes a sum at 4 TB/s.  Cut by 1 / 2 / 4:
            // 128 x 4096 x 4096 22.4 / 17.7 / 15.3 us, 256 x 8512 x 2048 16.5 / 22.0 / 27.7.
            auto tenths = [&](int64_t c) {
                const int64_t turns = (small * c + 3 * kComputeUnits - 1) / (3 * kComputeUnits);
                return (steps + c - 1) / c * 6 * turns + (c > 1 ? 40 + c * m * n * 8 / 400000 : 0);
            };
            for (int64_t c = 2; c <= 16 && c <= steps / 4; ++c)
                if (tenths(c) < tenths(slices)) slices = c;
        }
    }
    if (slices > 16) slices = 16;
    if (slices < 2) return s;
    s.slice_k = (int)((steps + slices - 1) / slices) * 128;
    s.slices = (int)((k + s.slice_k - 1) / s.slice_k);
    return s;
}

template <typename T, int BM, int BN, int WM, int WN, int STAGES, bool GROUPED, bool GATED> static int launch_q8(const Q8Args &q, hipStream_t st)
{
    const int out = GATED ? BN / 2 : BN;
    const int64_t tiles = GROUPED ? GroupedGrid(q.a, BM, out).tiles : ((int64_t)(q.a.m + BM - 1) / BM) * ((q.a.n + out - 1) / out);
    if (tiles * 64 * WM * WN >= 1ll << 32) return WPK_E_UNSUPPORTED;
    hipLaunchKernelGGL((linear_q8_kernel<T, BM, BN, WM, WN, STAGES, GROUPED, GATED>), dim3((unsigned)tiles, q.a.slices), dim3(64 * WM * WN), 0, st, q);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}
template <typename T, bool GROUPED, bool GATED> static int launch_q8_form(int form, const Q8Args &q, hipStream_t st)
{
    if constexpr (sizeof(T) == 2) {
        if (form == kQ8Tile256) return launch_q8<T, 256, 256, 2, 4, 2, GROUPED, GATED>(q, st);
        if (form == kQ8Tile128) return launch_q8<T, 128, 128, 2, 4, 2, GROUPED, GATED>(q, st);
    }
    return launch_q8<T, 64, 128, 1, 4, 2, GROUPED, GATED>(q, st);
}

template <typename T, int MT, int NT, bool GROUPED, bool GATED> static int launch_q8_rows(const Q8Args &q, int64_t tiles, hipStream_t st)
{
    const int U = MT == 4 || sizeof(T) == 4 ? 1 : 2;
    if (tiles * 64 * kRowsWaves >= 1ll << 32) return WPK_E_UNSUPPORTED;
    hipLaunchKernelGGL((linear_q8_rows_kernel<T, MT, NT, U, GROUPED, GATED>), dim3((unsigned)tiles, q.a.slices), dim3(64 * kRowsWaves), 0, st, q);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}
template <typename T, int MT> static int linear_q8_rows(const Q8Args &q, hipStream_t st)
{
    const int64_t tiles = (q.a.n + q.a.width - 1) / q.a.width;
    if (q.a.width <= 16) return launch_q8_rows<T, MT, 1, false, false>(q, tiles, st);
    if (q.a.width <= 32) return launch_q8_rows<T, MT, 2, false, false>(q, tiles, st);
    return launch_q8_rows<T, MT, 3, false, false>(q, tiles, st);
}

template <typename T> static int linear_q8_typed(const Q8Args &q, const Q8Shape &s, hipStream_t st)
{
    int rc;
    if (s.form == kQ8Rows) rc = q.a.m <= 16 ? linear_q8_rows<T, 1>(q, st) : q.a.m <= 32 ? linear_q8_rows<T, 2>(q, st) : linear_q8_rows<T, 4>(q, st);
    else rc = launch_q8_form<T, false, false>(s.form, q, st);
    if (rc != WPK_OK || s.slices == 1) return rc;
    const int64_t quads = (int64_t)((q.a.n + 3) / 4) * q.a.m;
    hipLaunchKernelGGL((linear_join_kernel<T>), dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, st, q.a);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

// us, rows kernel / tiles of 64 / 128 / 256, bf16 y, experts x columns x reduction (gated: twice the columns) and the mean of their
// rows, of uneven spread:
//   8 x 2048 x 2048:          mean 1: 9.5 / 18 / 22 / 40     16: 15 / 19 / 26 / 42     32: 27 / 19 / 26 / 43   512: - / 45 / 50 / 50
//   64 x 1024 x 2048, gated:  mean 1: 40 / 35 / 50 / 81      64: 294 / 74 / 81 / 120  128: 556 / 112 / 99 / 120   256: - / 176 / 146 / 130
//   128 x 768 x 1024, gated:  mean 4: 74 / 50 / 62 / 83      64: 312 / 69 / 72 / 105  128: 577 / 99 / 90 / 107    512: - / 285 / 227 / 213
template <typename T, bool GATED> static int grouped_q8_typed(Q8Args q, hipStream_t st)
{
    const int64_t rows = q.a.m, groups = q.a.groups, mean = rows / groups;
    q.a.width = GATED ? 16 : 32;
    // as many workgroups as the row kernel would have at the least
    const int64_t few = ((groups < rows ? groups : rows) + rows / 16) * ((q.a.n + q.a.width - 1) / q.a.width);
    if (few <= 4 * kComputeUnits) return launch_q8_rows<T, 1, 2, true, GATED>(q, GroupedGrid(q.a, 16, q.a.width).tiles, st);
    auto tiles = [&](int64_t m, int64_t n) { return rows / m * ((q.a.n + n - 1) / n); };
    const int form = q.a.k < 1024                                                               ? kQ8Tile64
                     : mean >= 256 && tiles(256, GATED ? 128 : 256) >= 2 * kComputeUnits        ? kQ8Tile256
                     : mean >= 128 && tiles(64, GATED ? 64 : 128) > 4 * kComputeUnits           ? kQ8Tile128
                                                                                                : kQ8Tile64;
    return launch_q8_form<T, true, GATED>(form, q, st);
}

int grouped_q8(const Q8Args &q, int y_dtype, bool gated, hipStream_t st)
{
    // Loads reach 2^31 bytes from the first row where rows are looked up or a weight has two halves.
    const int64_t far = 1ll << 31;
    if ((q.a.source && (q.a.x_rows * q.a.x_stride >= far || q.a.x_rows * q.x_scale_stride * 4 >= far)) || (gated && 2ll * q.a.n * q.a.w_stride >= far)) return WPK_E_UNSUPPORTED;
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
    const int rc = wpk::check_linear_q8(d);
    if (rc != WPK_OK) return rc;
    const wpk::Q8Shape s = wpk::q8_shape(d->m, d->n, d->k, d->dtype);
    return s.slices < 2 ? 0 : (int64_t)s.slices * d->m * (((int64_t)d->n + 3) / 4 * 4) * (int64_t)sizeof(float);
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
    const Q8Shape s = q8_shape(d.m, d.n, d.k, d.dtype);
    if (s.slices > 1 && !workspace) return WPK_E_NULL_PTR;
    const LinearArgs a = {x, w, bias, residual, y, (float *)workspace, d.m, d.n, d.k, d.act, d.dtype == WPK_F32, s.slices, s.slice_k,
                          s.width, wide, d.x_stride, d.w_stride, d.y_stride, d.residual_stride, ((int64_t)d.n + 3) / 4 * 4, nullptr, nullptr,
                          1, d.m, 0};
    const Q8Args q = {a, x_scales, w_scales, d.x_scale_stride, d.w_scale_stride, 0};
    const hipStream_t st = (hipStream_t)stream;
    if (d.dtype == WPK_BF16) return linear_q8_typed<bf16>(q, s, st);
    if (d.dtype == WPK_F16) return linear_q8_typed<f16>(q, s, st);
    return linear_q8_typed<float>(q, s, st);
}

}  // extern "C"
