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
    int32_t vec_bc, vec_x, vec_z, vec_y, vec_state;   // rows that vector accesses may be used on
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

template <int PARTS> __device__ inline void split(float v, bf16 (&out)[PARTS])
{
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        out[i] = (bf16)v;
        v -= (float)out[i];
    }
}

// Offset of the eight elements `chunk` of row `row` in a matrix of NCH such chunks a row.  Chunks are dealt out so that
// sixteen consecutive rows' same chunk covers all banks, and rows eight apart (transposing writes) half of them.
template <int NCH> __device__ inline int lds_at(int row, int chunk)
{
    const int f = NCH >= 16 ? (row ^ (row >> 4)) & 15 : NCH == 8 ? ((row >> 1) ^ (row >> 4)) & 7 : ((row >> 2) ^ (row >> 4)) & 3;
    return (row * NCH + (chunk ^ f)) * 8;
}

template <typename T, int V> struct Raw {
    typedef T vec __attribute__((ext_vector_type(V), aligned(V * sizeof(T) < 16 ? V * sizeof(T) : 16)));
    vec v;
    __device__ void load(const T *p, bool row_ok, int left, bool wide)   // left: columns from p on that exist
    {
        if (row_ok && wide && left > 0) {
            v = *(const vec *)p;
            return;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = row_ok && i < left ? p[i] : (T)0.0f;
    }
};

// One part of a request: FULL computes y and the state at its end, otherwise only what its tokens add to a state.
template <typename T, int NPAD, int Q, bool FULL> struct SsmScan {
    static const int NP = SsmType<T>::parts;
    static const int YP = NP == 3 ? 3 : 2;           // parts of what is formed on the way to y
    static const int NB = NPAD / 16, QB = Q / 16, QK = Q / 32, NCH = NPAD / 8, QCH = Q / 8;
    static const int kBTasks = (Q / 4) * NCH, kBPer = (kBTasks + 255) / 256;   // 4 tokens x 8 columns of B and C each
    static const int kXTasks = (Q / 4) * 16, kXPer = (kXTasks + 255) / 256;    // 4 tokens x 4 rows of X
    static const int kBlocks = Q == 64 ? 12 : 4;      // 16 x 16 blocks of M, those of zeros beside the diagonal included
    static const int kPerWave = kBlocks / 4;
    // M takes the place of B's rows where both do not fit a compute unit's LDS
    static const bool kAlias = NP * Q * NPAD * 6 + NP * 64 * Q * 2 + YP * Q * Q * 2 + 24 * Q > 163000;

    struct Shared {
        bf16 bt[NP][NPAD * Q];                        // [n][s]
        bf16 xt[NP][64 * Q];                          // [p][s]
        bf16 c[FULL ? NP : 1][FULL ? Q * NPAD : 8];   // [t][n]
        bf16 b[FULL ? NP : 1][FULL ? Q * NPAD : 8];   // [s][n]
        bf16 m[FULL && !kAlias ? YP : 1][FULL && !kAlias ? Q * Q : 8];   // [t][s]
        float sh[Q], sl[Q], delta[Q], into[Q], from[Q];   // S in two floats, delta, exp(S_end - S) delta, exp(S)
        float keep;
        int odd[2];                                   // a chunk holds infinities or NaN in x
    };

    static __device__ bf16 *m_at(Shared &sm, int part, int offset)
    {
        return kAlias ? &sm.b[0][part * Q * Q + offset] : &sm.m[kAlias ? 0 : part][offset];
    }

    static __device__ void run(const SsmArgs<T> &a, Shared &sm)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, g = lane >> 4;
        const int head = blockIdx.x % a.heads, pblock = blockIdx.x / a.heads, part = blockIdx.y, r = blockIdx.z;
        const int P = a.head_dim, N = a.state_dim, group = head / (a.heads / a.groups);
        int first, length;
        request_rows(a.rq, r, &first, &length);
        const int chunks = (length + Q - 1) / Q;
        // this part's chunks; a request has as many parts as it has chunks for, one at least
        const int parts = min(max((chunks + a.part_chunks - 1) / a.part_chunks, 1), a.n_parts);
        if (FULL ? part >= parts : part >= parts - 1) return;
        const int c0 = part * a.part_chunks, c1 = part == parts - 1 ? chunks : c0 + a.part_chunks;

        const int p_base = pblock * 64, p = p_base + wave * 16 + col;   // p: the state row whose columns this lane holds
        const int slot = request_slot(a.rq, r);
        const bool resume = a.state_in && slot >= 0 && (!a.rq.resume || a.rq.resume[r] != 0);
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
        // The state before the part.  Parts meet through the workspace: entry i holds what part i's tokens leave (part 0's
        // with the state before the request), the last entry the state before the request itself, since whoever does the
        // last part may be writing the pool's entry already.
        bool zero_state = true;
        if (part == 0) {
            if (resume) {
                add_state(FULL && parts > 1 ? ws + (size_t)(a.n_parts - 1) * state_size : a.state_in + pool_at, 0.0f);
                zero_state = false;
                if (!FULL) put_state(ws + (size_t)(a.n_parts - 1) * state_size);
            }
        } else if (FULL) {
            for (int i = 0; i < part; ++i) add_state(ws + (size_t)i * state_size, i ? a.part_decay[ws_head * a.n_parts + i] : 0.0f);
            zero_state = false;
        }

        const float rate = a.a[head], skip = a.d_skip ? a.d_skip[head] : 0.0f, dt_bias = a.dt_bias ? a.dt_bias[head] : 0.0f;
        const T *const bp = a.b + (int64_t)first * a.b_stride + group * N, *const cp = a.c + (int64_t)first * a.c_stride + group * N;
        const int64_t hp = (int64_t)head * P;
        const T *const xp = a.x + (int64_t)first * a.x_stride + hp, *const dtp = a.dt + (int64_t)first * a.dt_stride + head;

        Raw<T, 8> rb[kBPer][4], rc[FULL ? kBPer : 1][4];
        Raw<T, 4> rx[kXPer][4];
        float rdt = 0.0f;
        auto fetch = [&](int chunk) {
            const int t0 = chunk * Q;
#pragma unroll
            for (int i = 0; i < kBPer; ++i) {
                const int task = tid + 256 * i, n = (task % NCH) * 8, s = (task / NCH) * 4;
                if (kBTasks % 256 != 0 && task >= kBTasks) break;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int t = t0 + s + j;
                    rb[i][j].load(bp + (int64_t)t * a.b_stride + n, t < length, N - n, a.vec_bc);
                    if (FULL) rc[i][j].load(cp + (int64_t)t * a.c_stride + n, t < length, N - n, a.vec_bc);
                }
            }
#pragma unroll
            for (int i = 0; i < kXPer; ++i) {
                const int task = tid + 256 * i, q = p_base + (task % 16) * 4, s = (task / 16) * 4;
                if (kXTasks % 256 != 0 && task >= kXTasks) break;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int t = t0 + s + j;
                    rx[i][j].load(xp + (int64_t)t * a.x_stride + q, t < length, P - q, a.vec_x);
                }
            }
            if (tid < Q) rdt = t0 + tid < length ? (float)dtp[(int64_t)(t0 + tid) * a.dt_stride] : 0.0f;
        };
        auto stage = [&](int chunk) {
#pragma unroll
            for (int i = 0; i < kBPer; ++i) {
                const int task = tid + 256 * i, n = (task % NCH) * 8, s = (task / NCH) * 4;
                if (kBTasks % 256 != 0 && task >= kBTasks) break;
                bf16 v[4][8][NP];
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int k = 0; k < 8; ++k) split<NP>((float)rb[i][j].v[k], v[j][k]);
#pragma unroll
                for (int q = 0; q < NP; ++q) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const bf16x4 w = {v[0][k][q], v[1][k][q], v[2][k][q], v[3][k][q]};
                        *(bf16x4 *)&sm.bt[q][lds_at<QCH>(n + k, s >> 3) + (s & 7)] = w;
                    }
                    if (FULL)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            bf16x8 w;
#pragma unroll
                            for (int k = 0; k < 8; ++k) w[k] = v[j][k][q];
                            *(bf16x8 *)&sm.b[q][lds_at<NCH>(s + j, n >> 3)] = w;
                        }
                }
                if (FULL)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        bf16x8 w[NP];
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            bf16 u[NP];
                            split<NP>((float)rc[i][j].v[k], u);
#pragma unroll
                            for (int q = 0; q < NP; ++q) w[q][k] = u[q];
                        }
#pragma unroll
                        for (int q = 0; q < NP; ++q) *(bf16x8 *)&sm.c[q][lds_at<NCH>(s + j, n >> 3)] = w[q];
                    }
            }
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < kXPer; ++i) {
                const int task = tid + 256 * i, q4 = (task % 16) * 4, s = (task / 16) * 4;
                if (kXTasks % 256 != 0 && task >= kXTasks) break;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    bf16 v[4][NP];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float f = (float)rx[i][j].v[k];
                        sum = fmaf(f, 0.0f, sum);
                        split<NP>(f, v[j]);
                    }
#pragma unroll
                    for (int q = 0; q < NP; ++q) {
                        const bf16x4 w = {v[0][q], v[1][q], v[2][q], v[3][q]};
                        *(bf16x4 *)&sm.xt[q][lds_at<QCH>(q4 + k, s >> 3) + (s & 7)] = w;
                    }
                }
            }
            if (FULL && __any(sum != 0.0f) && lane == 0) sm.odd[chunk & 1] = 1;   // (NaN)
            if (wave == 0) {
                // lanes are tokens
                const bool live = lane < Q && chunk * Q + lane < length;
                float delta = rdt + dt_bias;
                if (a.softplus) delta = softplus(delta);
                if (!live) delta = 0.0f;
                double s = (double)delta * rate * 1.4426950408889634;
                if (s < -192.0) s = -192.0;
                if (!live) s = 0.0;
#pragma unroll
                for (int m = 1; m < Q; m <<= 1) {
                    const double o = __shfl_up(s, m);
                    if (lane >= m) s += o;
                }
                const double end = __shfl(s, Q - 1);
                if (lane < Q) {
                    sm.sh[lane] = (float)s;
                    sm.sl[lane] = (float)(s - (double)(float)s);
                    sm.delta[lane] = delta;
                    sm.into[lane] = delta * __builtin_amdgcn_exp2f((float)(end - s));
                    sm.from[lane] = __builtin_amdgcn_exp2f((float)s);
                }
                if (lane == 0) sm.keep = __builtin_amdgcn_exp2f((float)end);
            }
        };

        if (tid < 2) sm.odd[tid] = 0;
        float total = 1.0f;
        if (c0 < c1) fetch(c0);
        __syncthreads();
        for (int chunk = c0; chunk < c1; ++chunk) {
            stage(chunk);
            __syncthreads();
            const int t0 = chunk * Q;
            Raw<T, 4> rz[FULL ? QB : 1];
            const int p4 = p_base + wave * 16 + 4 * g;      // rows of y that this lane stores
            if (FULL && a.z)
#pragma unroll
                for (int i = 0; i < QB; ++i) {
                    const int t = t0 + 16 * i + col;
                    rz[i].load(a.z + (int64_t)(first + t) * a.z_stride + hp + p4, t < length, P - p4, a.vec_z);
                }
            if (chunk + 1 < c1) fetch(chunk + 1);
            if (tid == 0) sm.odd[(chunk + 1) & 1] = 0;
            const float keep = sm.keep;
            total *= keep;

            f32x4 acc[FULL ? QB : 1];
            if (FULL) {
                // G transposed, block by block (rows s, column t in the lane), into M
                f32x4 gt[kPerWave];
#pragma unroll
                for (int i = 0; i < kPerWave; ++i) {
                    const int k = wave + 4 * i, tb = k < 4 ? k >> 1 : 2 + ((k - 4) >> 2), sb = k < 4 ? k & 1 : (k - 4) & 3;
                    gt[i] = f32x4{0, 0, 0, 0};
                    if (sb > tb) continue;
#pragma unroll
                    for (int n = 0; n < NPAD / 32; ++n) {
                        bf16x8 fb[NP], fc[NP];
#pragma unroll
                        for (int q = 0; q < NP; ++q) {
                            fb[q] = *(const bf16x8 *)&sm.b[q][lds_at<NCH>(16 * sb + col, 4 * n + g)];
                            fc[q] = *(const bf16x8 *)&sm.c[q][lds_at<NCH>(16 * tb + col, 4 * n + g)];
                        }
                        gt[i] = mma_parts<NP>(fb, fc, gt[i]);
                    }
                }
                if (kAlias) __syncthreads();
#pragma unroll
                for (int i = 0; i < kPerWave; ++i) {
                    const int k = wave + 4 * i, tb = k < 4 ? k >> 1 : 2 + ((k - 4) >> 2), sb = k < 4 ? k & 1 : (k - 4) & 3;
                    const int t = 16 * tb + col, s0 = 16 * sb + 4 * g;
                    const f32x4 sh = *(const f32x4 *)&sm.sh[s0], sl = *(const f32x4 *)&sm.sl[s0], dl = *(const f32x4 *)&sm.delta[s0];
                    const float th = sm.sh[t], tl = sm.sl[t];
                    bf16x4 w[YP];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float v = gt[i][j] * (__builtin_amdgcn_exp2f((th - sh[j]) + (tl - sl[j])) * dl[j]);
                        if (s0 + j == t) v += skip;
                        if (s0 + j > t) v = 0.0f;
                        bf16 u[YP];
                        split<YP>(v, u);
#pragma unroll
                        for (int q = 0; q < YP; ++q) w[q][j] = u[q];
                    }
#pragma unroll
                    for (int q = 0; q < YP; ++q) *(bf16x4 *)m_at(sm, q, lds_at<QCH>(t, s0 >> 3) + (s0 & 7)) = w[q];
                }
                // exp(S) C h0: rows p, column t in the lane
#pragma unroll
                for (int i = 0; i < QB; ++i) acc[i] = f32x4{0, 0, 0, 0};
                if (!zero_state || chunk > c0) {
#pragma unroll
                    for (int n = 0; n < NPAD / 32; ++n) {
                        bf16x8 fh[YP];
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            bf16 u[YP];
                            split<YP>(h[2 * n + (j >> 2)][j & 3], u);
#pragma unroll
                            for (int q = 0; q < YP; ++q) fh[q][j] = u[q];
                        }
#pragma unroll
                        for (int i = 0; i < QB; ++i) {
                            bf16x8 fc[NP];
                            const int t = 16 * i + col;
#pragma unroll
                            for (int q = 0; q < NP; ++q) {
                                const bf16x4 lo = *(const bf16x4 *)&sm.c[q][lds_at<NCH>(t, 4 * n + (g >> 1)) + 4 * (g & 1)];
                                const bf16x4 hi = *(const bf16x4 *)&sm.c[q][lds_at<NCH>(t, 4 * n + 2 + (g >> 1)) + 4 * (g & 1)];
                                fc[q] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                            }
                            acc[i] = mma_parts<YP>(fh, fc, acc[i]);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < QB; ++i) acc[i] *= sm.from[16 * i + col];
                }
                __syncthreads();
            }

            bf16x8 fx[QK][NP];
#pragma unroll
            for (int k = 0; k < QK; ++k)
#pragma unroll
                for (int q = 0; q < NP; ++q) fx[k][q] = *(const bf16x8 *)&sm.xt[q][lds_at<QCH>(wave * 16 + col, 4 * k + g)];

            if (FULL) {
                if (!sm.odd[chunk & 1]) {
#pragma unroll
                    for (int i = 0; i < QB; ++i)
#pragma unroll
                        for (int k = 0; k <= i / 2; ++k) {
                            bf16x8 fm[YP];
#pragma unroll
                            for (int q = 0; q < YP; ++q)
                                fm[q] = *(const bf16x8 *)m_at(sm, q, lds_at<QCH>(16 * i + col, 4 * k + g));
                            acc[i] = mma_parts<YP>(fx[k], fm, acc[i]);
                        }
                } else {
                    // infinities or NaN among the chunk's x may not meet the zeros of M that stand for later tokens
#pragma unroll
                    for (int i = 0; i < QB; ++i) {
                        const int t = 16 * i + col;
                        for (int s = 0; s <= t; ++s) {
                            float m = 0.0f;
#pragma unroll
                            for (int q = 0; q < YP; ++q) m += (float)*m_at(sm, q, lds_at<QCH>(t, s >> 3) + (s & 7));
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                float x = 0.0f;
#pragma unroll
                                for (int q = 0; q < NP; ++q)
                                    x += (float)sm.xt[q][lds_at<QCH>(wave * 16 + 4 * g + j, s >> 3) + (s & 7)];
                                acc[i][j] = fmaf(m, x, acc[i][j]);
                            }
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < QB; ++i) {
                    const int t = t0 + 16 * i + col;
                    if (t >= length || p4 >= P) continue;
                    T *const yp = a.y + (int64_t)(first + t) * a.y_stride + hp + p4;
                    Raw<T, 4> out;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float v = acc[i][j];
                        if (a.z) v *= silu_as<T>((float)rz[i].v[j]);
                        out.v[j] = (T)v;
                    }
                    if (a.vec_y) *(typename Raw<T, 4>::vec *)yp = out.v;
                    else
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (p4 + j < P) yp[j] = out.v[j];
                }
            }

            // the state behind the chunk
            bf16x8 fw[QK][3];
#pragma unroll
            for (int k = 0; k < QK; ++k) {
                const f32x4 w0 = *(const f32x4 *)&sm.into[32 * k + 8 * g], w1 = *(const f32x4 *)&sm.into[32 * k + 8 * g + 4];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float x = 0.0f;
#pragma unroll
                    for (int q = NP - 1; q >= 0; --q) x += (float)fx[k][q][j];
                    bf16 u[3];
                    split<3>(x * (j < 4 ? w0[j & 3] : w1[j & 3]), u);
#pragma unroll
                    for (int q = 0; q < 3; ++q) fw[k][q][j] = u[q];
                }
            }
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                h[i] *= keep;
#pragma unroll
                for (int k = 0; k < QK; ++k) {
                    bf16x8 fb[NP];
#pragma unroll
                    for (int q = 0; q < NP; ++q) fb[q] = *(const bf16x8 *)&sm.bt[q][lds_at<QCH>(16 * i + col, 4 * k + g)];
                    h[i] = mma_parts<3>(fb, fw[k], h[i]);
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

template <typename T, int NPAD, int Q, bool FULL> __global__ void __launch_bounds__(256, (sizeof(typename SsmScan<T, NPAD, Q, FULL>::Shared) > 81920 ? 1 : 2))
ssm_scan_kernel(SsmArgs<T> a)
{
    typedef SsmScan<T, NPAD, Q, FULL> Scan;
    __shared__ typename Scan::Shared sm;
    Scan::run(a, sm);
}

}  // namespace wpk
#endif
