// Selective state space scan over prompts, in chunks of kQ tokens on the bf16 matrix pipes.
//
// With S the running sum of delta a within a chunk, h0 the state before it and G = C B^T:
//   M[t][s] = G[t][s] exp(S_t - S_s) delta_s  (s <= t; d on the diagonal too)     y = M X + exp(S_t) C h0
//   h1 = exp(S_end) h0 + sum_s B_s (outer) exp(S_end - S_s) delta_s x_s
// so a token costs products of matrices instead of a pass over the state: 2 Q N / P + Q + 4 N operations an element
// instead of 5 N on the vector units.
//
// A workgroup of four waves walks through the chunks of one head (64 rows of its state, 16 a wave) with the state in
// registers; nothing of it goes to memory between chunks.  All MFMAs are 16x16x32: the accumulators of h (column p in the
// lane, rows n four by four) are, taken two blocks at a time, what the next product's operand wants with its reduction index
// permuted, and C is read from LDS with the same permutation, so the state never crosses lanes either.  X stands in LDS
// transposed and B both ways, transposed in registers on the way in.
//
// Types.  Operands are taken as sums of bf16 numbers: one for bf16, two for fp16 (exact), three for fp32.  What is formed
// in fp32 on the way keeps two of them (2^-17 of it) where y is rounded to 16 bits, and three (all 24 bits) for fp32 and
// for what goes into the state, which stays fp32.  S is summed in 64 bits and kept as two floats: differences of far tokens
// would lose the small decays between them otherwise.  A token's delta a is held above -192 octaves, where exp is 0 in 32 bits.
#ifndef WPK_SSM_SCAN_H
#define WPK_SSM_SCAN_H

#include "wpk_seq.h"

namespace wpk {

template <typename T> struct SsmArgs {
    const T *x, *dt, *b, *c, *z;
    const float *a, *d_skip, *dt_bias, *state_in;
    float *state_out;
    T *y;
    Requests rq;
    int32_t heads, head_dim, groups, state_dim, softplus;
    int64_t x_stride, dt_stride, b_stride, c_stride, z_stride, y_stride;
    // prompts only
    float *parts;             // workspace: [request][head][parts][head_dim][state_dim], then [request][head][parts] decays
    float *part_decay;
    int32_t n_parts;          // parts that a request may have
    int32_t part_chunks;      // chunks of a part (the last one takes what is left)
    int32_t sequences;        // 0 where requests are done in their order, else as many, the longest first (256 at most)
    int32_t vec_rows, vec_state;   // whether rows (of the tensors, of the states) start at multiples of 16 bytes
};

template <typename T> struct SsmType;
template <> struct SsmType<bf16> { static const int parts = 1; };
template <> struct SsmType<f16> { static const int parts = 2; };
template <> struct SsmType<float> { static const int parts = 3; };

__device__ inline f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// sum over pairs of parts whose indexes add up to less than LIMIT
template <int LIMIT, int PA, int PB> __device__ inline f32x4 mma_parts(const bf16x8 (&a)[PA], const bf16x8 (&b)[PB], f32x4 c)
{
#pragma unroll
    for (int i = 0; i < PA; ++i)
#pragma unroll
        for (int j = 0; j < PB; ++j)
            if (i + j < LIMIT) c = mma(a[i], b[j], c);
    return c;
}

// the pairs that mma_parts takes, one by one, for products that are better interleaved
template <int LIMIT, int PA, int PB, typename F> __device__ inline void each_pair(F f)
{
#pragma unroll
    for (int i = 0; i < PA; ++i)
#pragma unroll
        for (int j = 0; j < PB; ++j)
            if (i + j < LIMIT) f(i, j);
}

// values as sums of parts, the largest first
template <typename BF, int PARTS, typename F> __device__ inline void split(F v, BF (&out)[PARTS])
{
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        out[i] = __builtin_convertvector(v, BF);
        if (i + 1 < PARTS) v -= __builtin_convertvector(out[i], F);
    }
}
template <int PARTS> __device__ inline void parts_of(bf16 v, bf16 (&out)[PARTS]) { out[0] = v; }
template <int PARTS, typename T> __device__ inline void parts_of(T v, bf16 (&out)[PARTS])
{
    float f = (float)v;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        out[i] = (bf16)f;
        f -= (float)out[i];
    }
}

// Number of the request that is longer than all but n (ties in their order), by one workgroup of 256 at least; `room` holds
// 257 numbers.  Long requests that start last would leave the device to themselves at the end.
__device__ inline int nth_longest(const Requests &q, int sequences, int n, int *room)
{
    const int i = threadIdx.x;
    if (i < sequences) {
        const int a = min(max(q.starts[i], 0), q.tokens), b = min(max(q.starts[i + 1], 0), q.tokens);
        room[i] = max(b - a, 0);
    }
    __syncthreads();
    if (i < sequences) {
        const int mine = room[i];
        int before = 0;
        for (int j = 0; j < sequences; ++j) before += room[j] > mine || (room[j] == mine && j < i);
        if (before == n) room[256] = i;
    }
    __syncthreads();
    const int r = __builtin_amdgcn_readfirstlane(room[256]);
    __syncthreads();
    return r;
}

// a request has as many parts as it has chunks for, one at least
template <typename T> __device__ inline int parts_of_request(const SsmArgs<T> &a, int chunks)
{
    return min(max((chunks + a.part_chunks - 1) / a.part_chunks, 1), a.n_parts);
}

// One part of a request: FULL computes y and the state at its end, otherwise only what its tokens add to a state.
template <typename T, int NPAD, int Q, bool FULL, bool WIDE> struct SsmScan {
    static const int NP = SsmType<T>::parts;
    static const int YP = NP == 3 ? 3 : 2;           // parts of what is formed on the way to y
    static const int NB = NPAD / 16, QB = Q / 16, QK = Q / 32, NCH = NPAD / 8, QCH = Q / 8;
    static const int kBTasks = (Q / 4) * NCH, kBPer = (kBTasks + 255) / 256;   // 4 tokens x 8 columns of B and C each
    static const int kXTasks = (Q / 4) * 16, kXPer = (kXTasks + 255) / 256;    // 4 tokens x 4 rows of X
    static const int kBlocks = Q == 64 ? 12 : 4;      // 16 x 16 blocks of M, those of zeros beside the diagonal included
    static const int kPerWave = kBlocks / 4;
    // M takes the place of B's rows where both do not fit a compute unit's LDS
    static const bool kAlias = NP * (2 * Q * (NPAD + 8) + (NPAD + 64) * (Q + 8)) * 2 + YP * Q * (Q + 8) * 2 + 48 * Q > 163000;

    // Rows of LDS matrices are eight elements longer than they have to be: the same columns of sixteen rows cover all banks.
    // (Of fp32's 256 columns only those of B and C are, and the scalars have one place, formed while chunks are staged.)
    static const bool kTight = NP == 3 && NPAD == 256;
    static const int kN = NPAD + 8, kS = kTight ? Q : Q + 8, kSc = kTight ? 1 : 2;
    // M holds columns up to the end of a row's 32 tokens only
    static const int kM = Q == 64 ? 32 * 40 + 32 * kS : Q * kS;
    static __device__ int m_row(int t) { return Q == 64 ? (t < 32 ? t * 40 : t * kS - 32 * (kS - 40)) : t * kS; }

    struct alignas(16) Scalars {
        // S in two floats, delta, exp(S_end - S) delta, exp(S), exp(S_e - S) delta with e the end of a token's block of 16
        alignas(16) float sh[Q], sl[Q], delta[Q], into[Q], from[Q], block[Q];
        float keep[4];
    };
    struct alignas(16) Shared {
        alignas(16) bf16 bt[NP][NPAD * kS];                       // [n][s]
        alignas(16) bf16 xt[NP][64 * kS];                         // [p][s]
        alignas(16) bf16 c[FULL ? NP : 1][FULL ? Q * kN : 8];     // [t][n]
        alignas(16) bf16 b[FULL ? NP : 1][FULL ? Q * kN : 8];     // [s][n]
        alignas(16) bf16 m[FULL && !kAlias ? YP : 1][FULL && !kAlias ? kM : 8];   // [t][s]
        Scalars sc[kSc];                              // of the even and the odd chunks
    };

    static __device__ bf16 *m_at(Shared &sm, int part, int offset)
    {
        return kAlias ? &sm.b[0][part * kM + offset] : &sm.m[kAlias ? 0 : part][offset];
    }

    // What a lane moves: four tokens s.. of eight columns of B and C, or of four rows of X.  Lanes of a wave are dealt out
    // over tokens and columns so that the transposing writes to LDS meet at most two to a bank.
    static __device__ void b_task(int task, int *s, int *chunk)
    {
        const int high = Q == 64 ? 2 : 1;
        *s = 4 * ((task & 3) | ((task >> 4) & ((1 << high) - 1)) << 2);
        *chunk = ((task >> 2) & 3) | (task >> (4 + high)) << 2;
    }
    static __device__ void x_task(int task, int *s, int *quad)
    {
        *s = 4 * (((task >> 2) & 7) | (Q == 64 ? ((task >> 6) & 1) << 3 : 0));
        *quad = (task & 3) | ((task >> 5) & 1) << 2 | (task >> (Q == 64 ? 7 : 6)) << 3;
    }

    static __device__ void run(const SsmArgs<T> &a, Shared &sm)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, g = lane >> 4;
        const int head = blockIdx.x % a.heads, pblock = blockIdx.x / a.heads, part = blockIdx.y;
        const int r = a.sequences ? nth_longest(a.rq, a.sequences, blockIdx.z, (int *)&sm.bt[0][0]) : blockIdx.z;
        const int P = a.head_dim, N = a.state_dim, group = head / (a.heads / a.groups);
        int first, length;
        request_rows(a.rq, r, &first, &length);
        const int chunks = (length + Q - 1) / Q;
        // this part's chunks
        const int parts = parts_of_request(a, chunks);
        if (FULL ? part >= parts : part >= parts - 1) return;
        const int c0 = part * a.part_chunks, c1 = part == parts - 1 ? chunks : c0 + a.part_chunks;

        const int p_base = pblock * 64, p = p_base + wave * 16 + col;   // p: the state row whose columns this lane holds
        const int slot = request_slot(a.rq, r);
        const bool resume = a.state_in && slot >= 0 && request_resumes(a.rq, r);
        const size_t state_size = (size_t)P * N, row_at = (size_t)min(p, P - 1) * N;
        const size_t pool_at = ((size_t)max(slot, 0) * a.heads + head) * state_size + row_at;
        const size_t ws_head = (size_t)r * a.heads + head;
        float *const ws = a.parts ? a.parts + ws_head * a.n_parts * state_size + row_at : nullptr;

        f32x4 h[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) h[i] = f32x4{0, 0, 0, 0};
        const bool has_row = p < P;
        auto add_state = [&](const float *src, float decay) {      // h = decay h + src
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int n = 16 * i + 4 * g;
                f32x4 v = {0, 0, 0, 0};
                if (has_row && n < N) {
                    if (a.vec_state) v = *(const f32x4 *)(src + n);
                    else
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (n + j < N) v[j] = src[n + j];
                }
                h[i] = h[i] * decay + v;
            }
        };
        auto put_state = [&](float *dst) {
            if (!has_row) return;
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int n = 16 * i + 4 * g;
                if (n >= N) continue;
                if (a.vec_state) *(f32x4 *)(dst + n) = h[i];
                else
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (n + j < N) dst[n + j] = h[i][j];
            }
        };
        // The state before the part.  Parts meet through the workspace: entry i holds the state behind part i (what its
        // tokens leave, until ssm_join_kernel has added what the parts before it left), the last entry the state before the
        // request itself, since whoever does the last part may be writing the pool's entry already.
        if (part == 0) {
            if (resume) {
                add_state(FULL && parts > 1 ? ws + (size_t)(a.n_parts - 1) * state_size : a.state_in + pool_at, 0.0f);
                if (!FULL) put_state(ws + (size_t)(a.n_parts - 1) * state_size);
            }
        } else if (FULL) {
            add_state(ws + (size_t)(part - 1) * state_size, 0.0f);
        }

        const float rate = a.a[head], skip = a.d_skip ? a.d_skip[head] : 0.0f, dt_bias = a.dt_bias ? a.dt_bias[head] : 0.0f;
        const T *const bp = a.b + (int64_t)first * a.b_stride + group * N, *const cp = a.c + (int64_t)first * a.c_stride + group * N;
        const int64_t hp = (int64_t)head * P;
        const T *const xp = a.x + (int64_t)first * a.x_stride + hp, *const dtp = a.dt + (int64_t)first * a.dt_stride + head;

        Piece<T, 8> rb[kBPer][4], rc[FULL ? kBPer : 1][4];
        Piece<T, 4> rx[kXPer][4];
        const uint32_t e = sizeof(T);
        const uint32_t bs = (uint32_t)a.b_stride * e, cs = (uint32_t)a.c_stride * e, xs = (uint32_t)a.x_stride * e;
        const uint32_t zs = (uint32_t)a.z_stride * e, ys = (uint32_t)a.y_stride * e;
        auto fetch = [&](int chunk, bool want_b, bool want_c, bool want_x) {
            const int t0 = chunk * Q, left = min(length - t0, Q);       // rows that there are
            const Rows brows = rows_at(bp + (int64_t)t0 * a.b_stride, left, bs), crows = rows_at(cp + (int64_t)t0 * a.c_stride, left, cs);
            const Rows xrows = rows_at(xp + (int64_t)t0 * a.x_stride, left, xs);
#pragma unroll
            for (int i = 0; i < kBPer; ++i) {
                int s, n;
                b_task(tid + 256 * i, &s, &n);
                const uint32_t out = 8 * n < N && s < Q ? 0 : kOutside;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (want_b) rb[i][j].template load<WIDE>(brows, (s * bs + n * 8 * e | out) + j * bs, N - 8 * n);
                    if (FULL && want_c) rc[i][j].template load<WIDE>(crows, (s * cs + n * 8 * e | out) + j * cs, N - 8 * n);
                }
            }
#pragma unroll
            for (int i = 0; i < kXPer; ++i) {
                int s, q;
                x_task(tid + 256 * i, &s, &q);
                q = p_base + 4 * q;
                const uint32_t out = q < P ? 0 : kOutside;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (want_x) rx[i][j].template load<WIDE>(xrows, (s * xs + q * e | out) + j * xs, P - q);
            }
        };
        auto stage = [&]() {
#pragma unroll
            for (int i = 0; i < kBPer; ++i) {
                int s, n;
                b_task(tid + 256 * i, &s, &n);
                if (kBTasks % 256 != 0 && tid + 256 * i >= kBTasks) continue;
                bf16 v[4][8][NP];
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int k = 0; k < 8; ++k) parts_of<NP>((T)rb[i][j].v[k], v[j][k]);
#pragma unroll
                for (int q = 0; q < NP; ++q) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const bf16x4 w = {v[0][k][q], v[1][k][q], v[2][k][q], v[3][k][q]};
                        *(bf16x4 *)&sm.bt[q][(8 * n + k) * kS + s] = w;
                    }
                    if (FULL)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            bf16x8 w;
#pragma unroll
                            for (int k = 0; k < 8; ++k) w[k] = v[j][k][q];
                            *(bf16x8 *)&sm.b[q][(s + j) * kN + 8 * n] = w;
                        }
                }
                if (FULL)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        bf16x8 w[NP];
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            bf16 u[NP];
                            parts_of<NP>((T)rc[i][j].v[k], u);
#pragma unroll
                            for (int q = 0; q < NP; ++q) w[q][k] = u[q];
                        }
#pragma unroll
                        for (int q = 0; q < NP; ++q) *(bf16x8 *)&sm.c[q][(s + j) * kN + 8 * n] = w[q];
                    }
            }
#pragma unroll
            for (int i = 0; i < kXPer; ++i) {
                int s, q4;
                x_task(tid + 256 * i, &s, &q4);
                if (kXTasks % 256 != 0 && tid + 256 * i >= kXTasks) continue;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    bf16 v[4][NP];
#pragma unroll
                    for (int j = 0; j < 4; ++j) parts_of<NP>((T)rx[i][j].v[k], v[j]);
#pragma unroll
                    for (int q = 0; q < NP; ++q) {
                        const bf16x4 w = {v[0][q], v[1][q], v[2][q], v[3][q]};
                        *(bf16x4 *)&sm.xt[q][(4 * q4 + k) * kS + s] = w;
                    }
                }
            }
        };
        // One wave forms a chunk's scalars, its lanes the tokens, while the others are at the chunk before.
        Piece<T, 1> rdt;         // (converted where it is used, so that nothing waits for it before)
        auto fetch_dt = [&](int chunk) {
            const int t0 = chunk * Q;
            const uint32_t ds = (uint32_t)a.dt_stride * e;
            rdt.template load<false>(rows_at(dtp + (int64_t)t0 * a.dt_stride, min(length - t0, Q), ds), lane * ds, 1);
        };
        auto scalars = [&](int chunk) {
            Scalars &sc = sm.sc[chunk & (kSc - 1)];
            const bool live = lane < Q && chunk * Q + lane < length;
            float delta = (float)rdt.v[0] + dt_bias;
            if (a.softplus) delta = softplus_fast(delta);
            if (!live) delta = 0.0f;
            double s = (double)delta * rate * 1.4426950408889634;
            s = running_sum(!live ? 0.0 : s < -192.0 ? -192.0 : s);
            const double end = read_lane(s, Q - 1);
            if (lane < Q) {
                sc.sh[lane] = (float)s;
                sc.sl[lane] = (float)(s - (double)(float)s);
                sc.delta[lane] = delta;
                sc.into[lane] = delta * __builtin_amdgcn_exp2f((float)(end - s));
                sc.from[lane] = __builtin_amdgcn_exp2f((float)s);
                sc.block[lane] = delta * __builtin_amdgcn_exp2f((float)(row_end(s) - s));
            }
            if (lane == 0) sc.keep[0] = __builtin_amdgcn_exp2f((float)end);
        };
        const int kScalarWave = 0;

        float total = 1.0f;
        if (c0 < c1) {
            fetch(c0, true, true, true);
            if (wave == kScalarWave) {
                fetch_dt(c0);
                scalars(c0);
                fetch_dt(c0 + 1);
            }
        }
        const int p4 = p_base + wave * 16 + 4 * g;      // rows of y that this lane stores
        const uint32_t out4 = p4 < P ? 0 : kOutside;
        const bf16x8 zero8 = {0, 0, 0, 0, 0, 0, 0, 0};
        // This wave's 16 x 16 blocks of M: one on the diagonal and up to two below it (rows 1 .. 3 of four share six).  Blocks
        // above it in a row's 32 columns stay zero.
        const int tb0 = Q == 64 ? wave : wave & 1;
        const int tb1 = Q == 64 ? (wave == 0 ? 3 : wave) : 1, sb1 = Q == 64 ? (wave == 0 ? 0 : wave - 1) : 0;
        const int tb2 = wave == 1 ? 2 : 3, sb2 = wave == 1 ? 0 : 1;
        const bool has0 = Q == 64 || wave < 2, has1 = Q == 64 || wave == 2, has2 = Q == 64 && (wave & 1);
        auto zero_blocks = [&]() {
            if (wave == (Q == 64 ? 0 : 3) || (Q == 64 && wave == 2)) {
                const int t = 16 * (Q == 64 ? wave : 0) + col, s0 = 16 * (Q == 64 ? wave + 1 : 1) + 4 * g;
                const bf16x4 w = {0, 0, 0, 0};
#pragma unroll
                for (int q = 0; q < YP; ++q) *(bf16x4 *)m_at(sm, q, m_row(t) + s0) = w;
            }
        };
        if (FULL && !kAlias) zero_blocks();
        for (int chunk = c0; chunk < c1; ++chunk) {
            stage();
            if (kTight && chunk > c0 && wave == kScalarWave) {
                scalars(chunk);
                fetch_dt(chunk + 1);
            }
            __syncthreads();
            const int t0 = chunk * Q, left = min(length - t0, Q);
            const Scalars &sc = sm.sc[chunk & (kSc - 1)];
            Piece<T, 4> rz[FULL ? QB : 1];
            if (FULL && a.z) {
                const Rows zrows = rows_at(a.z + (int64_t)(first + t0) * a.z_stride + hp, left, zs);
#pragma unroll
                for (int i = 0; i < QB; ++i)
                    rz[i].template load<WIDE>(zrows, (col * zs + p4 * e | out4) + 16 * i * zs, P - p4);
            }
            const int next = min(chunk + 1, c1 - 1);       // (the last chunk again behind the last)
            fetch(next, true, false, !FULL);
            const float keep = sc.keep[0];
            total *= keep;

            f32x4 acc[FULL ? QB : 1];
            if (FULL) {
                // G transposed, block by block (rows s, column t in the lane), into M
                f32x4 g0 = {0, 0, 0, 0}, g1 = g0, g2 = g0;
                auto block = [&](int t, int u, f32x4 sum) {
#pragma unroll
                    for (int n = 0; n < NPAD / 32; ++n) {
                        bf16x8 fb[NP], fc[NP];
#pragma unroll
                        for (int q = 0; q < NP; ++q) {
                            fb[q] = *(const bf16x8 *)&sm.b[q][(16 * u + col) * kN + 8 * g + 32 * n];
                            fc[q] = *(const bf16x8 *)&sm.c[q][(16 * t + col) * kN + 8 * g + 32 * n];
                        }
                        sum = mma_parts<NP>(fb, fc, sum);
                    }
                    return sum;
                };
                auto put_block = [&](int t, int s0, f32x4 v) {
                    bf16x4 w[YP];
                    split(v, w);
#pragma unroll
                    for (int q = 0; q < YP; ++q) *(bf16x4 *)m_at(sm, q, m_row(t) + s0) = w[q];
                };
                // below the diagonal exp(S_t - S_s) is exp(S_t - S_e) exp(S_e - S_s), e the last token of the column's block
                auto below = [&](int tb, int sb, f32x4 v) {
                    const int t = 16 * tb + col, s0 = 16 * sb + 4 * g, end = 16 * sb + 15;
                    const float u = __builtin_amdgcn_exp2f((sc.sh[t] - sc.sh[end]) + (sc.sl[t] - sc.sl[end]));
                    put_block(t, s0, v * (*(const f32x4 *)&sc.block[s0] * u));
                };
                if (has0) g0 = block(tb0, tb0, g0);
                if (has1) g1 = block(tb1, sb1, g1);
                if (has2) g2 = block(tb2, sb2, g2);
                if (kAlias) {
                    __syncthreads();
                    zero_blocks();
                }
                if (has0) {
                    const int t = 16 * tb0 + col, s0 = 16 * tb0 + 4 * g;
                    const f32x4 sh = *(const f32x4 *)&sc.sh[s0], sl = *(const f32x4 *)&sc.sl[s0];
                    const f32x4 dl = *(const f32x4 *)&sc.delta[s0];
                    const float th = sc.sh[t], tl = sc.sl[t];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        g0[j] *= __builtin_amdgcn_exp2f((th - sh[j]) + (tl - sl[j])) * dl[j];
                        g0[j] = 4 * g + j > col ? 0.0f : 4 * g + j == col ? g0[j] + skip : g0[j];
                    }
                    put_block(t, s0, g0);
                }
                if (has1) below(tb1, sb1, g1);
                if (has2) below(tb2, sb2, g2);
                fetch(next, false, true, false);
                // exp(S) C h0: rows p, column t in the lane
#pragma unroll
                for (int i = 0; i < QB; ++i) acc[i] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int n = 0; n < NPAD / 32; ++n) {
                    bf16x8 fh[YP], fc[QB][NP];
                    split(__builtin_shufflevector(h[2 * n], h[2 * n + 1], 0, 1, 2, 3, 4, 5, 6, 7), fh);
#pragma unroll
                    for (int i = 0; i < QB; ++i)
#pragma unroll
                        for (int q = 0; q < NP; ++q) {
                            const bf16 *const at = &sm.c[q][(16 * i + col) * kN + 32 * n + 4 * g];
                            const bf16x4 lo = *(const bf16x4 *)at, hi = *(const bf16x4 *)(at + 16);
                            fc[i][q] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                        }
                    each_pair<YP, YP, NP>([&](int u, int v) {
#pragma unroll
                        for (int i = 0; i < QB; ++i) acc[i] = mma(fh[u], fc[i][v], acc[i]);
                    });
                }
#pragma unroll
                for (int i = 0; i < QB; ++i) acc[i] *= sc.from[16 * i + col];
            }
            if (!kTight && wave == kScalarWave && chunk + 1 < c1) {
                scalars(chunk + 1);
                fetch_dt(chunk + 2);
            }
            if (FULL) {
                __syncthreads();
                fetch(next, false, false, true);
            }

            bf16x8 fx[QK][NP];
#pragma unroll
            for (int k = 0; k < QK; ++k)
#pragma unroll
                for (int q = 0; q < NP; ++q) fx[k][q] = *(const bf16x8 *)&sm.xt[q][(wave * 16 + col) * kS + 32 * k + 8 * g];
            // Infinities or NaN among x may not meet the zeros of M that stand for later tokens: x times zero finds them.
            f32x4 odd = {0, 0, 0, 0};
            if (FULL)
#pragma unroll
                for (int k = 0; k < QK; ++k) odd = mma(fx[k][0], zero8, odd);

            // the state behind the chunk
#pragma unroll
            for (int i = 0; i < NB; ++i) h[i] *= keep;
#pragma unroll
            for (int k = 0; k < QK; ++k) {
                const f32x4 w0 = *(const f32x4 *)&sc.into[32 * k + 8 * g], w1 = *(const f32x4 *)&sc.into[32 * k + 8 * g + 4];
                f32x8 x = __builtin_convertvector(fx[k][NP - 1], f32x8);
#pragma unroll
                for (int q = NP - 2; q >= 0; --q) x += __builtin_convertvector(fx[k][q], f32x8);
                bf16x8 fw[3];
                split(x * __builtin_shufflevector(w0, w1, 0, 1, 2, 3, 4, 5, 6, 7), fw);
                const int kStep = NB * NP > 16 ? NB / 2 : NB;      // blocks of the state that go side by side
#pragma unroll
                for (int i0 = 0; i0 < NB; i0 += kStep) {
                    bf16x8 fb[kStep][NP];
#pragma unroll
                    for (int i = 0; i < kStep; ++i)
#pragma unroll
                        for (int q = 0; q < NP; ++q)
                            fb[i][q] = *(const bf16x8 *)&sm.bt[q][(16 * (i0 + i) + col) * kS + 32 * k + 8 * g];
                    each_pair<3, NP, 3>([&](int u, int v) {
#pragma unroll
                        for (int i = 0; i < kStep; ++i) h[i0 + i] = mma(fb[i][u], fw[v], h[i0 + i]);
                    });
                }
            }

            if (FULL) {
                if (!__any(odd[0] != 0.0f || odd[1] != 0.0f || odd[2] != 0.0f || odd[3] != 0.0f)) {
#pragma unroll
                    for (int k = 0; k < QK; ++k) {
                        bf16x8 fm[QB][YP];
#pragma unroll
                        for (int i = 2 * k; i < QB; ++i)
#pragma unroll
                            for (int q = 0; q < YP; ++q)
                                fm[i][q] = *(const bf16x8 *)m_at(sm, q, m_row(16 * i + col) + 32 * k + 8 * g);
                        each_pair<YP, NP, YP>([&](int u, int v) {
#pragma unroll
                            for (int i = 2 * k; i < QB; ++i) acc[i] = mma(fx[k][u], fm[i][v], acc[i]);
                        });
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < QB; ++i) {
                        const int t = 16 * i + col;
#pragma unroll 1
                        for (int s = 0; s <= t; ++s) {
                            float m = 0.0f;
#pragma unroll
                            for (int q = 0; q < YP; ++q) m += (float)*m_at(sm, q, m_row(t) + s);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                float x = 0.0f;
#pragma unroll
                                for (int q = 0; q < NP; ++q) x += (float)sm.xt[q][(wave * 16 + 4 * g + j) * kS + s];
                                acc[i][j] = fmaf(m, x, acc[i][j]);
                            }
                        }
                    }
                }
                const Rows yrows = rows_at(a.y + (int64_t)(first + t0) * a.y_stride + hp, left, ys);
#pragma unroll
                for (int i = 0; i < QB; ++i) {
                    Piece<T, 4> out;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float v = acc[i][j];
                        if (a.z) v *= silu_as<T>((float)rz[i].v[j]);
                        out.v[j] = (T)v;
                    }
                    out.template store<WIDE>(yrows, (col * ys + p4 * e | out4) + 16 * i * ys, P - p4);
                }
            }
            __syncthreads();
        }
        if (!FULL) {
            put_state(ws + (size_t)part * state_size);
            if (pblock == 0 && tid == 0) a.part_decay[ws_head * a.n_parts + part] = total;
        } else if (part == parts - 1 && a.state_out && slot >= 0) {
            put_state(a.state_out + pool_at);
        }
    }
};

template <typename T, int NPAD, int Q, bool FULL, bool WIDE>
__global__ void __launch_bounds__(256, (sizeof(typename SsmScan<T, NPAD, Q, FULL, WIDE>::Shared) > 81920 ? 1 : 2))
ssm_scan_kernel(SsmArgs<T> a)
{
    typedef SsmScan<T, NPAD, Q, FULL, WIDE> Scan;
    __shared__ typename Scan::Shared sm;
    Scan::run(a, sm);
}

// From what the parts' tokens leave to the states behind the parts: entry i of the workspace += decay of part i times entry
// i - 1, a lane to four numbers of a state.
template <typename T, int Q> __global__ void __launch_bounds__(256) ssm_join_kernel(SsmArgs<T> a)
{
    const int head = blockIdx.y, r = blockIdx.z;
    int first, length;
    request_rows(a.rq, r, &first, &length);
    const int parts = parts_of_request(a, (length + Q - 1) / Q);
    const int64_t size = (int64_t)a.head_dim * a.state_dim, at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (parts < 3 || at >= size) return;
    const int64_t ws_head = (int64_t)r * a.heads + head;
    float *const ws = a.parts + ws_head * a.n_parts * size + at;
    const float *const decay = a.part_decay + ws_head * a.n_parts;
    if (a.vec_state) {
        f32x4 cur = *(const f32x4 *)ws;
        for (int i = 1; i < parts - 1; i += 4) {
            f32x4 e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) e[j] = *(const f32x4 *)(ws + min(i + j, parts - 2) * size);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (i + j >= parts - 1) break;
                cur = cur * decay[i + j] + e[j];
                *(f32x4 *)(ws + (i + j) * size) = cur;
            }
        }
    } else {
        for (int c = 0; c < 4 && at + c < size; ++c) {
            float cur = ws[c];
            for (int i = 1; i < parts - 1; ++i) ws[i * size + c] = cur = cur * decay[i] + ws[i * size + c];
        }
    }
}

}  // namespace wpk
#endif
