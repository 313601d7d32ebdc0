// Selective state space scan over prompts (wpk_ssm_scan.h has the formulas): bf16, four heads of a group at a time.
//
// Heads of a group share B and C, and a wave that owns 32 rows of a state instead of 16 reads what it multiplies with from LDS
// half as often a row; LDS traffic and what goes into it are what bounds the form with one head a workgroup.  So here a
// workgroup of eight waves walks four "units" (64 rows of a head's state each) of one group through a part's chunks, two
// waves a unit, 32 rows a wave.  G = C B^T is formed by each half of the workgroup for its two units.  Operands whose reduction
// runs along the tokens (B and X, which stand in LDS as they stand in memory) are read with the transposing LDS read: sixteen
// lanes address four rows of sixteen columns and get a column's four entries each.  B and C go from memory to LDS directly, a
// chunk ahead.  The 16-byte pieces of a row stand in the order of their number xor some bits of the row's, so that both
// sixteen rows' same piece and four rows' neighbouring pieces lie in different banks.
#ifndef WPK_SSM_GROUP_H
#define WPK_SSM_GROUP_H

#include "wpk_ssm_scan.h"

namespace wpk {

// What is xored to the number of a 16-byte piece in a row of NCH pieces; the same for rows 32 apart.
template <int NCH> __device__ inline int piece_order(int row)
{
    return NCH >= 16 ? (row & 15) ^ ((row >> 4) & 1) << 2 : NCH == 8 ? ((row >> 1) & 7) ^ ((row >> 4) & 1) << 1 : (row >> 2) & 3;
}
template <int NCH> __device__ inline int piece_at(int row, int piece) { return (row * NCH + (piece ^ piece_order<NCH>(row))) * 8; }

typedef short s16x4 __attribute__((ext_vector_type(4)));
__device__ inline bf16x4 read_transposed(const bf16 *p)
{
    return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p));
}

template <int NPAD, bool FULL> struct GroupScan {
    typedef bf16 T;
    static const int Q = 64, NB = NPAD / 16, NCH = NPAD / 8, kThreads = 512, kUnits = 4;
    static const int kM = 32 * 32 + 32 * 64;             // columns of M up to the end of a row's 32 tokens

    struct alignas(16) Scalars {
        alignas(16) float sh[Q], sl[Q], delta[Q], into[Q], from[Q], block[Q];     // as in SsmScan
        float keep[4];
    };
    struct alignas(16) Shared {
        alignas(16) bf16 b[2][Q * NPAD];
        alignas(16) bf16 c[FULL ? 2 : 1][FULL ? Q * NPAD : 8];
        alignas(16) bf16 x[kUnits][Q * 64];
        alignas(16) bf16 m[FULL ? kUnits : 1][2][FULL ? kM : 8];
        Scalars sc[2][kUnits];
    };
    static __device__ int m_at(int t, int s)             // s a multiple of four
    {
        const int p = t < 32 ? (t * 4 + ((s >> 3) ^ ((t >> 2) & 3))) * 8 : 1024 + ((t - 32) * 8 + ((s >> 3) ^ ((t >> 1) & 7))) * 8;
        return p + (s & 4);
    }

    static __device__ void run(const SsmArgs<T> &a, Shared &sm)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        int lane_col = lane & 15, lane_g = lane >> 4;
        const int part = blockIdx.y, P = a.head_dim, N = a.state_dim;
        const int r = a.sequences ? nth_longest(a.rq, a.sequences, blockIdx.z, (int *)&sm.b[0][0]) : blockIdx.z;
        int first, length;
        request_rows(a.rq, r, &first, &length);
        const int chunks = (length + Q - 1) / Q, parts = parts_of_request(a, chunks);
        if (FULL ? part >= parts : part >= parts - 1) return;
        const int c0 = part * a.part_chunks, c1 = part == parts - 1 ? chunks : c0 + a.part_chunks;

        // units of a group: its heads' blocks of 64 rows; behind the last one the last again, without a trace
        const int each = a.heads / a.groups, blocks = (P + 63) / 64, units = each * blocks, teams = (units + kUnits - 1) / kUnits;
        const int group = blockIdx.x / teams, unit0 = (blockIdx.x - group * teams) * kUnits;
        auto head_of = [&](int u) { return group * each + min(unit0 + u, units - 1) / blocks; };
        auto block_of = [&](int u) { return min(unit0 + u, units - 1) % blocks; };
        const int unit = wave >> 1, head = head_of(unit), p_base = block_of(unit) * 64 + (wave & 1) * 32;
        const bool real = unit0 + unit < units;

        const int slot = request_slot(a.rq, r);
        const bool resume = a.state_in && slot >= 0 && request_resumes(a.rq, r);
        const size_t state_size = (size_t)P * N, pool_at = ((size_t)max(slot, 0) * a.heads + head) * state_size;
        const size_t ws_head = (size_t)r * a.heads + head;
        float *const ws = a.parts ? a.parts + ws_head * a.n_parts * state_size : nullptr;

        // states: rows n 16 i + 4 g .. + 3 of column p_base + 16 rb + col
        f32x4 h[2][NB];
        auto state_offset = [&](int rb, int i) -> uint32_t {
            const int p = p_base + 16 * rb + lane_col, n = 16 * i + 4 * lane_g;
            return p < P && n < N ? (uint32_t)(p * N + n) * 4 : kOutside;
        };
        auto get_state = [&](const float *src, bool there) {
            const Rows rows = rows_at(src, there ? 1 : 0, (uint32_t)state_size * 4);
#pragma unroll
            for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    Piece<float, 4> v;
                    v.template load<true>(rows, state_offset(rb, i), 4);
                    h[rb][i] = v.v;
                }
        };
        auto put_state = [&](float *dst, bool there) {
            const Rows rows = rows_at(dst, there && real ? 1 : 0, (uint32_t)state_size * 4);
#pragma unroll
            for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    Piece<float, 4> v;
                    v.v = h[rb][i];
                    v.template store<true>(rows, state_offset(rb, i), 4);
                }
        };
        // (as in SsmScan: entry i of the workspace is the state behind part i, the last one that before the request)
        if (part == 0) {
            float *const before = ws + (size_t)(a.n_parts - 1) * state_size;
            get_state(FULL && parts > 1 ? before : a.state_in + pool_at, resume);
            if (!FULL) put_state(before, resume);
        } else {
            get_state(ws + (size_t)(part - 1) * state_size, FULL);
        }

        const uint32_t e = sizeof(T);
        const uint32_t bs = (uint32_t)a.b_stride * e, cs = (uint32_t)a.c_stride * e, xs = (uint32_t)a.x_stride * e;
        const uint32_t zs = (uint32_t)a.z_stride * e, ys = (uint32_t)a.y_stride * e, ds = (uint32_t)a.dt_stride * e;
        const T *const bp = a.b + (int64_t)first * a.b_stride + group * N, *const cp = a.c + (int64_t)first * a.c_stride + group * N;
        const T *const xp = a.x + (int64_t)first * a.x_stride;

        // B and C, a load a wave bringing 1024 bytes of whole rows
        const int kLoads = NPAD / 8, kLoadRows = 512 / NPAD;
        auto fetch_rows = [&](int chunk) {
            const int t0 = chunk * Q, left = min(length - t0, Q);
#pragma unroll
            for (int w = 0; w < (FULL ? 2 : 1); ++w) {
                const Rows rows = w == 0 ? rows_at(bp + (int64_t)t0 * a.b_stride, left, bs) : rows_at(cp + (int64_t)t0 * a.c_stride, left, cs);
                const uint32_t to = lds_offset(w == 0 ? &sm.b[chunk & 1][0] : &sm.c[FULL ? chunk & 1 : 0][0]);
#pragma unroll
                for (int l0 = 0; l0 < kLoads; l0 += 8) {
                    const int l = l0 + wave, row = l * kLoadRows + lane / NCH, piece = lane % NCH ^ piece_order<NCH>(row);
                    if (kLoads < 8 && l >= kLoads) break;
                    load_to_lds(rows, piece * 8 < N ? row * (w == 0 ? bs : cs) + piece * 16 : kOutside, 0, to + l * 1024);
                }
            }
        };
        // X: four pieces a lane, of one unit
        const int x_unit = (tid & 31) >> 3, x_piece = tid & 7, x_p = block_of(x_unit) * 64 + x_piece * 8;
        const uint32_t x_off = x_p < P ? (uint32_t)(head_of(x_unit) * P + x_p) * e : kOutside;
        Piece<T, 8> rx[4];
        auto fetch_x = [&](int chunk) {
            const int t0 = chunk * Q;
            const Rows rows = rows_at(xp + (int64_t)t0 * a.x_stride, min(length - t0, Q), xs);
#pragma unroll
            for (int i = 0; i < 4; ++i) rx[i].template load<true>(rows, x_off + ((tid >> 5) + 16 * i) * xs, 8);
        };
        auto stage_x = [&]() {
#pragma unroll
            for (int i = 0; i < 4; ++i) *(bf16x8 *)&sm.x[x_unit][piece_at<8>((tid >> 5) + 16 * i, x_piece)] = rx[i].v;
        };
        // Waves 0, 2, 4 and 6 form the scalars of a unit each, a chunk ahead.
        const bool scalar_wave = (wave & 1) == 0;
        const float rate = a.a[head], dt_bias = a.dt_bias ? a.dt_bias[head] : 0.0f;
        Piece<T, 1> rdt;
        auto fetch_dt = [&](int chunk) {
            const int t0 = chunk * Q;
            rdt.template load<false>(rows_at(a.dt + (int64_t)(first + t0) * a.dt_stride + head, min(length - t0, Q), ds), lane * ds, 1);
        };
        auto scalars = [&](int chunk) {
            Scalars &sc = sm.sc[chunk & 1][unit];
            const bool live = chunk * Q + lane < length;
            float delta = (float)rdt.v[0] + dt_bias;
            if (a.softplus) delta = softplus_fast(delta);
            if (!live) delta = 0.0f;
            double s = (double)delta * rate * 1.4426950408889634;
            s = running_sum(!live ? 0.0 : s < -192.0 ? -192.0 : s);
            const double end = read_lane(s, Q - 1);
            sc.sh[lane] = (float)s;
            sc.sl[lane] = (float)(s - (double)(float)s);
            sc.delta[lane] = delta;
            sc.into[lane] = delta * __builtin_amdgcn_exp2f((float)(end - s));
            sc.from[lane] = __builtin_amdgcn_exp2f((float)s);
            sc.block[lane] = delta * __builtin_amdgcn_exp2f((float)(row_end(s) - s));
            if (lane == 0) sc.keep[0] = __builtin_amdgcn_exp2f((float)end);
        };

        // blocks of M, dealt out to the four waves of a half as in SsmScan
        const int w4 = wave & 3, pair = (wave >> 2) * 2;
        const int tb1 = w4 == 0 ? 3 : w4, sb1 = w4 == 0 ? 0 : w4 - 1, tb2 = w4 == 1 ? 2 : 3, sb2 = w4 == 1 ? 0 : 1;
        const bool has2 = w4 & 1;
        if (FULL && (w4 == 0 || w4 == 2)) {
            const bf16x4 w = {0, 0, 0, 0};
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int q = 0; q < 2; ++q) *(bf16x4 *)&sm.m[FULL ? pair + u : 0][q][m_at(16 * w4 + lane_col, 16 * (w4 + 1) + 4 * lane_g)] = w;
        }
        const int kNext = 8 * (NCH >= 16 ? 4 : NCH == 8 ? 2 : 1), kOdd = 8 * (NCH >= 16 ? 4 : NCH == 8 ? 2 : 0);

        float total = 1.0f;
        if (c0 < c1) {
            fetch_rows(c0);
            fetch_x(c0);
            if (scalar_wave) {
                fetch_dt(c0);
                scalars(c0);
                fetch_dt(c0 + 1);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        const bf16x8 zero8 = {0, 0, 0, 0, 0, 0, 0, 0};
        for (int chunk = c0; chunk < c1; ++chunk) {
            stage_x();
            __syncthreads();
            const int t0 = chunk * Q, left = min(length - t0, Q), next = min(chunk + 1, c1 - 1), cur = chunk & 1;
            const Scalars &sc = sm.sc[cur][unit];
            if (chunk + 1 < c1) fetch_rows(chunk + 1);
            // Offsets are formed anew for every chunk: kept over the loop, they would take the registers of half a state.
            asm volatile("" : "+v"(lane_col), "+v"(lane_g));
            const int col = lane_col, g = lane_g;
            // Where this lane's first pieces are: of four rows for the transposing reads of B (blocks of 16 columns) and X, of
            // rows t of C.  Other pieces of a row are at that xor 8 times theirs; rows 4 on (a second transposing read) and 16
            // on (C's odd blocks) differ from it by one bit of the order.
            const int trow = 8 * g + (col >> 2), half4 = (col & 1) * 4;
            const int at_b = piece_at<NCH>(trow, (col >> 1) & 1) + half4, at_c = piece_at<NCH>(col, g >> 1) + 4 * (g & 1);
            const int at_x = piece_at<8>(trow, 4 * (wave & 1) + ((col >> 1) & 1)) + half4;
            const float keep = sc.keep[0];
            total *= keep;

            f32x4 acc[2][4];
            if (FULL) {
                const bf16 *const bm = &sm.b[cur][0], *const cm = &sm.c[FULL ? cur : 0][0];
                f32x4 g0 = {0, 0, 0, 0}, g1 = g0, g2 = g0;
                auto block = [&](int t, int s, f32x4 sum) {
                    const int tr = 16 * t + col, sr = 16 * s + col, to = piece_order<NCH>(tr), so = piece_order<NCH>(sr);
#pragma unroll
                    for (int n = 0; n < NPAD / 32; ++n)
                        sum = mma(*(const bf16x8 *)(bm + (sr * NCH + ((4 * n + g) ^ so)) * 8),
                                  *(const bf16x8 *)(cm + (tr * NCH + ((4 * n + g) ^ to)) * 8), sum);
                    return sum;
                };
                auto put_block = [&](int u, int t, int s0, f32x4 v) {
                    bf16x4 w[2];
                    split(v, w);
#pragma unroll
                    for (int q = 0; q < 2; ++q) *(bf16x4 *)&sm.m[FULL ? u : 0][q][m_at(t, s0)] = w[q];
                };
                auto below = [&](int tb, int sb, f32x4 v) {
                    const int t = 16 * tb + col, s0 = 16 * sb + 4 * g, end = 16 * sb + 15;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const Scalars &q = sm.sc[cur][pair + u];
                        const float d = __builtin_amdgcn_exp2f((q.sh[t] - q.sh[end]) + (q.sl[t] - q.sl[end]));
                        put_block(pair + u, t, s0, v * (*(const f32x4 *)&q.block[s0] * d));
                    }
                };
                g0 = block(w4, w4, g0);
                g1 = block(tb1, sb1, g1);
                if (has2) g2 = block(tb2, sb2, g2);
                const int t = 16 * w4 + col, s0 = 16 * w4 + 4 * g;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const Scalars &q = sm.sc[cur][pair + u];
                    const float skip = a.d_skip ? a.d_skip[head_of(pair + u)] : 0.0f;
                    const f32x4 sh = *(const f32x4 *)&q.sh[s0], sl = *(const f32x4 *)&q.sl[s0], dl = *(const f32x4 *)&q.delta[s0];
                    const float th = q.sh[t], tl = q.sl[t];
                    f32x4 v;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        v[j] = g0[j] * (__builtin_amdgcn_exp2f((th - sh[j]) + (tl - sl[j])) * dl[j]);
                        v[j] = 4 * g + j > col ? 0.0f : 4 * g + j == col ? v[j] + skip : v[j];
                    }
                    put_block(pair + u, t, s0, v);
                }
                below(tb1, sb1, g1);
                if (has2) below(tb2, sb2, g2);

                // exp(S) C h0: rows p, column t in the lane
#pragma unroll
                for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[rb][i] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int n = 0; n < NPAD / 32; ++n) {
                    bf16x8 fh[2][2], fc[4];
#pragma unroll
                    for (int rb = 0; rb < 2; ++rb)
                        split(__builtin_shufflevector(h[rb][2 * n], h[rb][2 * n + 1], 0, 1, 2, 3, 4, 5, 6, 7), fh[rb]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int at = at_c ^ 32 * n ^ (i & 1 ? kOdd : 0);
                        const bf16x4 lo = *(const bf16x4 *)(cm + 16 * i * NPAD + at), hi = *(const bf16x4 *)(cm + 16 * i * NPAD + (at ^ 16));
                        fc[i] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    }
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                            for (int i = 0; i < 4; ++i) acc[rb][i] = mma(fh[rb][u], fc[i], acc[rb][i]);
                    __builtin_amdgcn_sched_barrier(0);         // (here and below: operands read further ahead do not fit the registers)
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float from = sc.from[16 * i + col];
                    acc[0][i] *= from;
                    acc[1][i] *= from;
                }
            }
            if (scalar_wave && chunk + 1 < c1) {
                scalars(chunk + 1);
                fetch_dt(chunk + 2);
            }
            if (FULL) __syncthreads();
            Piece<T, 4> rz[2][4];
            const int p4 = p_base + 4 * g;
            if (FULL) {
                const Rows zrows = rows_at(a.z + (int64_t)(first + t0) * a.z_stride + (int64_t)head * P, a.z ? left : 0, zs);
#pragma unroll
                for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        rz[rb][i].template load<true>(zrows, (col * zs + (p4 + 16 * rb) * e | (p4 + 16 * rb < P ? 0 : kOutside)) + 16 * i * zs, 4);
            }

            bf16x8 fx[2][2];
            const bf16 *const xm = &sm.x[unit][0];
#pragma unroll
            for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const bf16x4 lo = read_transposed(xm + 32 * k * 64 + (at_x ^ 16 * rb));
                    const bf16x4 hi = read_transposed(xm + (32 * k + 4) * 64 + (at_x ^ 16 * rb ^ 16));
                    fx[rb][k] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                }
            // (infinities or NaN among x may not meet the zeros of M that stand for later tokens: x times zero finds them)
            f32x4 odd[2];
#pragma unroll
            for (int rb = 0; rb < 2; ++rb) odd[rb] = mma(fx[rb][1], zero8, mma(fx[rb][0], zero8, f32x4{0, 0, 0, 0}));

            // the state behind the chunk
            const bf16 *const bm = &sm.b[cur][0];
#pragma unroll
            for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                for (int i = 0; i < NB; ++i) h[rb][i] *= keep;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const f32x4 w0 = *(const f32x4 *)&sc.into[32 * k + 8 * g], w1 = *(const f32x4 *)&sc.into[32 * k + 8 * g + 4];
                const f32x8 w = __builtin_shufflevector(w0, w1, 0, 1, 2, 3, 4, 5, 6, 7);
                bf16x8 fw[2][3];
#pragma unroll
                for (int rb = 0; rb < 2; ++rb) split(__builtin_convertvector(fx[rb][k], f32x8) * w, fw[rb]);
                const int kStep = NB < 4 ? NB : 4;
#pragma unroll
                for (int i0 = 0; i0 < NB; i0 += kStep) {
                    bf16x8 fb[kStep];
#pragma unroll
                    for (int i = 0; i < kStep; ++i) {
                        const bf16x4 lo = read_transposed(bm + 32 * k * NPAD + (at_b ^ 16 * (i0 + i)));
                        const bf16x4 hi = read_transposed(bm + (32 * k + 4) * NPAD + (at_b ^ 16 * (i0 + i) ^ kNext));
                        fb[i] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    }
#pragma unroll
                    for (int v = 0; v < 3; ++v)
#pragma unroll
                        for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                            for (int i = 0; i < kStep; ++i) h[rb][i0 + i] = mma(fb[i], fw[rb][v], h[rb][i0 + i]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }

            fetch_x(next);
            if (FULL) {
                bool bad = false;
#pragma unroll
                for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                    for (int j = 0; j < 4; ++j) bad = bad || odd[rb][j] != 0.0f;
                if (!__any(bad)) {
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int i = 2 * k; i < 4; ++i)
#pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                const bf16x8 fm = *(const bf16x8 *)&sm.m[FULL ? unit : 0][q][m_at(16 * i + col, 32 * k + 8 * g)];
#pragma unroll
                                for (int rb = 0; rb < 2; ++rb) acc[rb][i] = mma(fx[rb][k], fm, acc[rb][i]);
                            }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int t = 16 * i + col;
#pragma unroll 1
                        for (int s = 0; s <= t; ++s) {
                            const int at = m_at(t, s & ~3) + (s & 3);
                            const float m = (float)sm.m[FULL ? unit : 0][0][at] + (float)sm.m[FULL ? unit : 0][1][at];
#pragma unroll
                            for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    const int p = (wave & 1) * 32 + 16 * rb + 4 * g + j;
                                    acc[rb][i][j] = fmaf(m, (float)xm[piece_at<8>(s, p >> 3) + (p & 7)], acc[rb][i][j]);
                                }
                        }
                    }
                }
                // the next chunk's rows are in LDS before y goes out
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                const Rows yrows = rows_at(a.y + (int64_t)(first + t0) * a.y_stride + (int64_t)head * P, real ? left : 0, ys);
#pragma unroll
                for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        Piece<T, 4> out;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float v = acc[rb][i][j];
                            if (a.z) v *= silu_as<T>((float)rz[rb][i].v[j]);
                            out.v[j] = (T)v;
                        }
                        out.template store<true>(yrows, (col * ys + (p4 + 16 * rb) * e | (p4 + 16 * rb < P ? 0 : kOutside)) + 16 * i * ys, 4);
                    }
            } else {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
            __syncthreads();
        }
        asm volatile("" : "+v"(lane_col), "+v"(lane_g));
        if (!FULL) {
            put_state(ws + (size_t)part * state_size, true);
            if (real && block_of(unit) == 0 && (wave & 1) == 0 && lane == 0) a.part_decay[ws_head * a.n_parts + part] = total;
        } else if (part == parts - 1) {
            put_state(a.state_out + pool_at, a.state_out && slot >= 0);
        }
    }
};

template <int NPAD, bool FULL> __global__ void __launch_bounds__(512, 2) ssm_group_kernel(SsmArgs<bf16> a)
{
    typedef GroupScan<NPAD, FULL> Scan;
    __shared__ typename Scan::Shared sm;
    Scan::run(a, sm);
}

}  // namespace wpk
#endif
