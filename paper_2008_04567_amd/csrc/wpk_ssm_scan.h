// Selective state space scan over prompts, in chunks of Q tokens on the bf16 matrix pipes.
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
// permuted, and C is read from LDS with the same permutation, so the state never crosses lanes either.  B, C and X stand in
// LDS as they come, once: what the other products want transposed is read by the transposing reads.  The order of a row's
// 16-byte pieces depends on the row, so that neither whole pieces nor transposing reads meet a bank twice.  The next chunk's rows come into
// registers while this one is worked on.
//
// No unit is busy all the time: 16384 tokens of 32 heads of 64 x 128 numbers, bf16, take 119 us in this pass (kernels alone,
// under a profiler), the vector units busy for 50 % of it, LDS for 35 % (a third of that conflicts, from C's reads, which the
// compiler joins two rows apart by 16 to one), the matrix pipes for 19 %, and waves wait for 24 % of theirs.  A chunk of 64 tokens
// costs a wave some 910 vector instructions (decays, splitting into parts, offsets), 113 of LDS and 102 MFMAs between its
// barriers, and a SIMD has two waves to fill them.  The pass that leaves the parts' states takes 47 us, their join 8.
//
// Two workgroups a compute unit with all operands under way in registers.  Measured on the way here, all kernels of such a call
// summed under the profiler: three workgroups, with rows fetched late, 178 us instead of 170; a wave that forms the next chunk's
// decays beside the others' products 175; transposed copies of B and X in LDS, written on the way in, 168, but 259 instead of 247
// for 24 ragged requests.  Four heads of a group in a workgroup, sharing G, took as long as one by one.  (A head of other than 64
// rows shares worse: of 32, two waves of four multiply zeros, 268 us instead of 152 for twice as many heads; of 128, two
// workgroups form the same G, 152 us for half as many.)
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
    int32_t part_chunks;      // chunks of a part (the last one takes what is left); before the launch: units of 64 tokens
    int32_t sequences;        // 0 where requests are done in their order, else as many, the longest first (256 at most)
    // whether rows of the tensors start at multiples of four bytes and hold whole groups of eight; of the states, at multiples of
    // 16 bytes
    int32_t vec_rows, vec_state;
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

// What is xored to the number of a 16-byte piece in a row of NCH pieces; the same for rows 16 apart.  Reads of one piece of 16
// rows meet every bank once, and so do transposing reads, whose half a wave takes 32 bytes (two pieces) of rows r .. r + 3
// and r + 8 .. r + 11, r a multiple of four.
template <int NCH> __device__ inline int piece_order(int row)
{
    const int pair = NCH >= 16 ? (row & 3) | (row >> 1 & 4) : NCH == 8 ? (row >> 1 & 1) | (row >> 2 & 2) : row >> 3 & 1;
    return pair << 1 | (row >> 2 & 1);
}
template <int NCH> __device__ inline int piece_at(int row, int piece) { return (row * NCH + (piece ^ piece_order<NCH>(row))) * 8; }

typedef short s16x4 __attribute__((ext_vector_type(4)));
__device__ inline bf16x4 read_transposed(const bf16 *p)
{
    return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p));
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
__device__ inline int parts_of_request(int part_chunks, int n_parts, int chunks)
{
    return min(max((chunks + part_chunks - 1) / part_chunks, 1), n_parts);
}

// One part of a request: FULL computes y and the state at its end, otherwise only what its tokens add to a state.
template <typename T, int NPAD, int Q, bool FULL, bool WIDE> struct SsmScan {
    static const int NP = SsmType<T>::parts;
    static const int YP = NP == 3 ? 3 : 2;           // parts of what is formed on the way to y
    static const int NB = NPAD / 16, QB = Q / 16, QK = Q / 32, NCH = NPAD / 8;
    static const int kBPer = (Q * NCH + 255) / 256;  // pieces of eight columns of a row that a lane moves, of B and of C
    static const int kXPer = Q * 8 / 256;            // and of X
    static const int kM = Q == 64 ? 32 * 32 + 32 * 64 : 32 * 32;      // columns of M up to the end of a row's 32 tokens

    struct alignas(16) Shared {
        alignas(16) bf16 b[NP][Q * NPAD];             // [s][n]
        alignas(16) bf16 x[NP][Q * 64];               // [s][p]
        alignas(16) bf16 c[FULL ? NP : 1][FULL ? Q * NPAD : 8];      // [t][n]
        alignas(16) bf16 m[FULL ? YP : 1][FULL ? kM : 8];            // [t][s]
        // of the chunk's tokens: S in two floats, delta, exp(S_end - S) delta, exp(S_e - S) delta with e the end of a token's
        // block of 16
        alignas(16) float sh[Q], sl[Q], delta[Q], into[Q], block[Q];
        float keep;
    };
    static __device__ int m_at(int t, int s)          // s a multiple of four
    {
        const int p = t < 32 ? (t * 4 + ((s >> 3) ^ ((t >> 2) & 3))) * 8 : 1024 + ((t - 32) * 8 + ((s >> 3) ^ ((t >> 1) & 7))) * 8;
        return p + (s & 4);
    }

    // The kernel's arguments where the launch left them, read again from there: what only a part's end wants would otherwise be
    // kept in registers that its chunks have a use for.
    typedef const __attribute__((address_space(4))) SsmArgs<T> *Again;
    static __device__ Again arguments_again()
    {
        uint64_t at = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(at));
        return (Again)at;
    }

    // where this workgroup's part is
    struct Part {
        int head, part, parts, first, length, c0, c1, slot, p;      // p: the lane's row of the head's state
        bool resume;
        size_t pool_at, ws_head;
        float *ws;
    };
    template <typename A> static __device__ Part locate(A a, int r)
    {
        const Requests rq = {a->rq.starts, a->rq.slot_map, a->rq.resume, a->rq.tokens, a->rq.max_length, a->rq.slots};
        Part w;
        w.head = blockIdx.x % a->heads;
        w.part = blockIdx.y;
        request_rows(rq, r, &w.first, &w.length);
        const int chunks = (w.length + Q - 1) / Q;
        w.parts = parts_of_request(a->part_chunks, a->n_parts, chunks);
        w.c0 = w.part * a->part_chunks;
        w.c1 = w.part == w.parts - 1 ? chunks : w.c0 + a->part_chunks;
        w.p = blockIdx.x / a->heads * 64 + (threadIdx.x >> 6) * 16 + (threadIdx.x & 15);
        w.slot = request_slot(rq, r);
        w.resume = a->state_in && w.slot >= 0 && request_resumes(rq, r);
        const size_t size = (size_t)a->head_dim * a->state_dim;
        w.pool_at = ((size_t)max(w.slot, 0) * a->heads + w.head) * size;
        w.ws_head = (size_t)r * a->heads + w.head;
        w.ws = a->parts ? a->parts + w.ws_head * a->n_parts * size : nullptr;
        return w;
    }

    // the state: rows n 16 i + 4 g .. + 3 of column p (its row of the head's 64)
    template <typename A> static __device__ void get_state(A a, int p, f32x4 (&h)[NB], const float *src, bool there)
    {
        const int P = a->head_dim, N = a->state_dim, g = threadIdx.x >> 4 & 3;
        const Rows rows = rows_at(src, there ? 1 : 0, (uint32_t)(P * N) * 4);
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int n = 16 * i + 4 * g, left = p < P ? N - n : 0;
            const uint32_t at = (uint32_t)(p * N + n) * 4;
            Piece<float, 4> v;
            if (a->vec_state) v.template load<true>(rows, left > 0 ? at : kOutside, 4);
            else v.template load<false>(rows, at, left);
            h[i] = v.v;
        }
    }
    template <typename A> static __device__ void put_state(A a, int p, const f32x4 (&h)[NB], float *dst, bool there)
    {
        const int P = a->head_dim, N = a->state_dim, g = threadIdx.x >> 4 & 3;
        const Rows rows = rows_at(dst, there ? 1 : 0, (uint32_t)(P * N) * 4);
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int n = 16 * i + 4 * g, left = p < P ? N - n : 0;
            const uint32_t at = (uint32_t)(p * N + n) * 4;
            Piece<float, 4> v;
            v.v = h[i];
            if (a->vec_state) v.template store<true>(rows, left > 0 ? at : kOutside, 4);
            else v.template store<false>(rows, at, left);
        }
    }

    // The state before the part.  Parts meet through the workspace: entry i holds the state behind part i (what its tokens
    // leave, until ssm_join_kernel has added what the parts before it left), the last entry the state before the request itself,
    // since whoever does the last part may be writing the pool's entry already.
    template <typename A> static __device__ void get_before(A a, const Part &w, f32x4 (&h)[NB])
    {
        const size_t size = (size_t)a->head_dim * a->state_dim;
        if (w.part > 0) get_state(a, w.p, h, w.ws + (size_t)(w.part - 1) * size, FULL);
        else get_state(a, w.p, h, FULL && w.parts > 1 ? w.ws + (size_t)(a->n_parts - 1) * size : a->state_in + w.pool_at, w.resume);
    }

    // rows of W columns, `cols` of them there, as they are
    template <int W> static __device__ void stage_plain(T *to, const T *from, int64_t stride, int cols, int left)
    {
        const Rows rows = rows_at(from, left, (uint32_t)stride * sizeof(T));
        for (int task = threadIdx.x; task < Q * W / 8; task += 256) {
            const int row = task / (W / 8), n = task % (W / 8) * 8;
            Piece<T, 8> v;
            v.template load<WIDE>(rows, n < cols ? (row * (uint32_t)stride + n) * sizeof(T) : kOutside, cols - n);
            __builtin_memcpy(__builtin_assume_aligned(&to[row * W + n], 16), &v.v, sizeof(v.v));
        }
    }

    // The part again as the definition has it, token by token in 32 bits: for values that the products cannot carry.  A wave
    // has its 16 rows of the state as before (`mine`: unless nothing happened to them), rows of B, C and X stand in LDS as they
    // come, and of four tokens at a time lane group g gates and stores the g-th.  One request of 16384 tokens of 32 heads of 64 x
    // 128 numbers, bf16, with an infinity among its first: 1380 us.
    static __device__ void walk(Again a, const Part &w, Shared &sm, bool mine, f32x4 (&h)[NB])
    {
        const int P = a->head_dim, N = a->state_dim, head = w.head, group = head / (a->heads / a->groups);
        const int p_base = blockIdx.x / a->heads * 64, tid = threadIdx.x;
        int g = tid >> 4 & 3;
        const uint32_t e = sizeof(T), zs = (uint32_t)a->z_stride * e, ys = (uint32_t)a->y_stride * e;
        const float rate = a->a[head], skip = a->d_skip ? a->d_skip[head] : 0.0f, dt_bias = a->dt_bias ? a->dt_bias[head] : 0.0f;
        const int64_t hp = (int64_t)head * P;
        typedef T tvec __attribute__((ext_vector_type(4)));
        T *const lb = (T *)&sm.b[0][0], *const lc = (T *)&sm.c[0][0], *const lx = (T *)&sm.x[0][0];
        static_assert(sizeof(sm.b) >= Q * NPAD * sizeof(T) && sizeof(sm.x) >= Q * 64 * sizeof(T), "room for plain rows");
        static_assert(!FULL || sizeof(sm.c) >= Q * NPAD * sizeof(T), "room for plain rows");
#pragma unroll 1
        for (int chunk = w.c0; chunk < w.c1; ++chunk) {
            const int left = min(w.length - chunk * Q, Q);
            const int64_t t0 = w.first + chunk * Q;
            stage_plain<NPAD>(lb, a->b + t0 * a->b_stride + group * N, a->b_stride, N, left);
            if (FULL) stage_plain<NPAD>(lc, a->c + t0 * a->c_stride + group * N, a->c_stride, N, left);
            stage_plain<64>(lx, a->x + t0 * a->x_stride + hp + p_base, a->x_stride, P - p_base, left);
            if (tid < Q) {                           // (tokens that are not there change nothing)
                float delta = 0.0f;
                if (tid < left) {
                    delta = (float)a->dt[(t0 + tid) * a->dt_stride + head] + dt_bias;
                    if (a->softplus) delta = softplus(delta);
                }
                sm.delta[tid] = delta;
                sm.into[tid] = tid < left ? expf(delta * rate) : 1.0f;       // (what a token keeps, here)
            }
            __syncthreads();
            const Rows zrows = rows_at(a->z + t0 * a->z_stride + hp, FULL && a->z ? left : 0, zs);
            const Rows yrows = rows_at(a->y + t0 * a->y_stride + hp, left, ys);
            const uint32_t at_p = w.p < P ? w.p * e : kOutside;
            Piece<T, 1> z, next, y;
            next.template load<false>(zrows, at_p + g * zs, FULL);
#pragma unroll 1
            for (int t4 = 0; mine && t4 < left; t4 += 4) {
                z = next;
                if (FULL) next.template load<false>(zrows, at_p + (t4 + 4 + g) * zs, 1);
                float sums[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    asm volatile("" : "+v"(g));      // (which numbers there are is found anew for every token, not held for all)
                    const int t = t4 + u;
                    const float keep = sm.into[t], in_x = sm.delta[t] * (float)lx[t * 64 + w.p - p_base];
                    float s = 0.0f;
#pragma unroll
                    for (int k = 0; k < NB; ++k) {
                        const int n = 16 * k + 4 * g;
                        const tvec b = *(const tvec *)&lb[t * NPAD + n];
                        h[k] = h[k] * keep + __builtin_convertvector(b, f32x4) * in_x;
                        if constexpr (FULL) {
                            const f32x4 c = __builtin_convertvector(*(const tvec *)&lc[t * NPAD + n], f32x4);
                            f32x4 v = h[k] * c;
#pragma unroll
                            for (int j = 1; j < 4 && !WIDE; ++j) v[j] = n + j < N ? v[j] : 0.0f;
                            s += n < N ? (v[0] + v[1]) + (v[2] + v[3]) : 0.0f;       // (elsewhere infinities would meet zeros)
                        }
                        if (NB * sizeof(T) > 16 && k % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                    }
                    sums[u] = s;
                }
                if constexpr (FULL) {
                    // lane group g gets the whole of the g-th sum
                    const bool g0 = g & 1, g1 = g & 2;
                    float s01 = g0 ? sums[1] : sums[0], s23 = g0 ? sums[3] : sums[2];
                    s01 += __shfl_xor(g0 ? sums[0] : sums[1], 16);
                    s23 += __shfl_xor(g0 ? sums[2] : sums[3], 16);
                    float s = g1 ? s23 : s01;
                    s += __shfl_xor(g1 ? s01 : s23, 32);
                    if (a->d_skip) s += skip * (float)lx[(t4 + g) * 64 + w.p - p_base];
                    if (a->z) s *= silu_as<T>((float)z.v[0]);
                    y.v[0] = (T)s;
                    y.template store<false>(yrows, at_p + (t4 + g) * ys, 1);
                }
            }
            __syncthreads();
        }
    }

    static __device__ void run(const SsmArgs<T> &a, Shared &sm)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        int lane_col = lane & 15, lane_g = lane >> 4;
        const int r = a.sequences ? nth_longest(a.rq, a.sequences, blockIdx.z, (int *)&sm.b[0][0]) : blockIdx.z;
        const Part w = locate(&a, r);
        if (FULL ? w.part >= w.parts : w.part >= w.parts - 1) return;
        const int head = w.head, first = w.first, length = w.length, c0 = w.c0, c1 = w.c1;
        const int P = a.head_dim, N = a.state_dim, group = head / (a.heads / a.groups), p_base = blockIdx.x / a.heads * 64;
        f32x4 h[NB];
        get_before(&a, w, h);
        if (!FULL && w.part == 0) put_state(&a, w.p, h, w.ws + (size_t)(a.n_parts - 1) * P * N, w.resume);

        const float rate = a.a[head], skip = a.d_skip ? a.d_skip[head] : 0.0f, dt_bias = a.dt_bias ? a.dt_bias[head] : 0.0f;
        const int64_t hp = (int64_t)head * P;
        const T *const bp = a.b + (int64_t)first * a.b_stride + group * N, *const cp = a.c + (int64_t)first * a.c_stride + group * N;
        const T *const xp = a.x + (int64_t)first * a.x_stride + hp, *const dtp = a.dt + (int64_t)first * a.dt_stride + head;
        const uint32_t e = sizeof(T);
        const uint32_t bs = (uint32_t)a.b_stride * e, cs = (uint32_t)a.c_stride * e, xs = (uint32_t)a.x_stride * e;
        const uint32_t zs = (uint32_t)a.z_stride * e, ys = (uint32_t)a.y_stride * e, ds = (uint32_t)a.dt_stride * e;

        // A chunk's rows are held in registers while the chunk before is worked on, and cut into their parts on the way to LDS.
        Piece<T, 8> rb[kBPer], rc[FULL ? kBPer : 1], rx[kXPer];
        Piece<T, 1> rdt;
        auto fetch_rows = [&](Piece<T, 8> *held, const T *from, int64_t stride, uint32_t bytes, int chunk) {
            const Rows rows = rows_at(from + (int64_t)chunk * Q * stride, min(length - chunk * Q, Q), bytes);
#pragma unroll
            for (int i = 0; i < kBPer; ++i) {
                const int task = tid + 256 * i, row = task / NCH, n = task % NCH * 8;
                held[i].template load<WIDE>(rows, n < N ? row * bytes + n * e : kOutside, n < N ? N - n : 0);
            }
        };
        auto fetch_x = [&](int chunk) {
            const Rows rows = rows_at(xp + (int64_t)chunk * Q * a.x_stride, min(length - chunk * Q, Q), xs);
#pragma unroll
            for (int i = 0; i < kXPer; ++i) {
                const int p = p_base + (tid & 7) * 8, row = (tid >> 3) + 32 * i;
                rx[i].template load<WIDE>(rows, p < P ? row * xs + p * e : kOutside, p < P ? P - p : 0);
            }
            if (wave == 0) rdt.template load<false>(rows_at(dtp + (int64_t)chunk * Q * a.dt_stride, min(length - chunk * Q, Q), ds), lane * ds, 1);
        };
        auto put_piece = [&](bf16 (&to)[NP][Q * NPAD], int at, const Piece<T, 8> &v) {
            bf16x8 w[NP];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                bf16 u[NP];
                parts_of<NP>((T)v.v[k], u);
#pragma unroll
                for (int q = 0; q < NP; ++q) w[q][k] = u[q];
            }
#pragma unroll
            for (int q = 0; q < NP; ++q) *(bf16x8 *)&to[q][at] = w[q];
        };
        auto stage = [&]() {
#pragma unroll
            for (int i = 0; i < kBPer; ++i) {
                const int task = tid + 256 * i, at = piece_at<NCH>(task / NCH, task % NCH);
                if (Q * NCH % 256 != 0 && task >= Q * NCH) continue;
                put_piece(sm.b, at, rb[i]);
                if constexpr (FULL) put_piece(sm.c, at, rc[i]);
            }
#pragma unroll
            for (int i = 0; i < kXPer; ++i) {
                bf16x8 w[NP];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    bf16 u[NP];
                    parts_of<NP>((T)rx[i].v[k], u);
#pragma unroll
                    for (int q = 0; q < NP; ++q) w[q][k] = u[q];
                }
#pragma unroll
                for (int q = 0; q < NP; ++q) *(bf16x8 *)&sm.x[q][piece_at<8>((tid >> 3) + 32 * i, tid & 7)] = w[q];
            }
        };
        // lanes are tokens
        auto scalars = [&](int chunk) {
            const bool live = lane < Q && chunk * Q + lane < length;
            float delta = (float)rdt.v[0] + dt_bias;
            if (a.softplus) delta = softplus_fast(delta);
            if (!live) delta = 0.0f;
            double s = (double)delta * rate * 1.4426950408889634;
            s = running_sum(!live ? 0.0 : s < -192.0 ? -192.0 : s);
            const double end = read_lane(s, Q - 1);
            if (lane < Q) {
                sm.sh[lane] = (float)s;
                sm.sl[lane] = (float)(s - (double)(float)s);
                sm.delta[lane] = delta;
                sm.into[lane] = delta * __builtin_amdgcn_exp2f((float)(end - s));
                sm.block[lane] = delta * __builtin_amdgcn_exp2f((float)(row_end(s) - s));
            }
            if (lane == 0) sm.keep = __builtin_amdgcn_exp2f((float)end);
        };

        // This wave's 16 x 16 blocks of M: one on the diagonal and up to two below it (rows 1 .. 3 of four share six).  Blocks
        // above it in a row's 32 columns stay zero.
        const int tb0 = Q == 64 ? wave : wave & 1;
        const int tb1 = Q == 64 ? (wave == 0 ? 3 : wave) : 1, sb1 = Q == 64 ? (wave == 0 ? 0 : wave - 1) : 0;
        const int tb2 = wave == 1 ? 2 : 3, sb2 = wave == 1 ? 0 : 1;
        const bool has0 = Q == 64 || wave < 2, has1 = Q == 64 || wave == 2, has2 = Q == 64 && (wave & 1);
        if (FULL && (wave == (Q == 64 ? 0 : 3) || (Q == 64 && wave == 2))) {
            const int t = 16 * (Q == 64 ? wave : 0) + lane_col, s0 = 16 * (Q == 64 ? wave + 1 : 1) + 4 * lane_g;
            const bf16x4 w = {0, 0, 0, 0};
#pragma unroll
            for (int q = 0; q < YP; ++q) *(bf16x4 *)&sm.m[FULL ? q : 0][m_at(t, s0)] = w;
        }

        float total = 1.0f;
        if (c0 < c1) {
            fetch_rows(rb, bp, a.b_stride, bs, c0);
            if constexpr (FULL) fetch_rows(rc, cp, a.c_stride, cs, c0);
            fetch_x(c0);
        }
        float odd = 0.0f;                                // NaN once there was an infinity or NaN in y before its gate
        for (int chunk = c0; chunk < c1; ++chunk) {
            stage();
            if (wave == 0) scalars(chunk);
            __syncthreads();
            const int t0 = chunk * Q, left = min(length - t0, Q), next = min(chunk + 1, c1 - 1);   // (the last chunk again behind it)
            // Offsets are formed anew for every chunk: kept over the loop, they would take registers of operands under way.
            asm volatile("" : "+v"(lane_col), "+v"(lane_g));
            const int col = lane_col, g = lane_g;
            // Where this lane's first pieces are: of four rows for the transposing reads of B (blocks of 16 columns) and X, of
            // rows t of C.  Other pieces of a row are at that xor 8 times theirs, and in rows 4 on (a second
            // transposing read) at that xor 8.
            const int trow = 8 * g + (col >> 2), half4 = (col & 1) * 4;
            const int at_b = piece_at<NCH>(trow, (col >> 1) & 1) + half4, at_c = piece_at<NCH>(col, g >> 1) + 4 * (g & 1);
            const int at_x = piece_at<8>(trow, 2 * wave + ((col >> 1) & 1)) + half4;
            const float keep = sm.keep;
            total *= keep;
            fetch_rows(rb, bp, a.b_stride, bs, next);

            f32x4 acc[FULL ? QB : 1];
            if constexpr (FULL) {
                // G transposed, block by block (rows s, column t in the lane), into M
                f32x4 g0 = {0, 0, 0, 0}, g1 = g0, g2 = g0;
                auto block = [&](int t, int s, f32x4 sum) {
                    const int tr = 16 * t + col, sr = 16 * s + col, to = piece_order<NCH>(tr), so = piece_order<NCH>(sr);
#pragma unroll
                    for (int n = 0; n < NPAD / 32; ++n) {
                        bf16x8 fb[NP], fc[NP];
#pragma unroll
                        for (int q = 0; q < NP; ++q) {
                            fb[q] = *(const bf16x8 *)&sm.b[q][(sr * NCH + ((4 * n + g) ^ so)) * 8];
                            fc[q] = *(const bf16x8 *)&sm.c[q][(tr * NCH + ((4 * n + g) ^ to)) * 8];
                        }
                        sum = mma_parts<NP>(fb, fc, sum);
                    }
                    return sum;
                };
                auto put_block = [&](int t, int s0, f32x4 v) {
                    bf16x4 w[YP];
                    split(v, w);
#pragma unroll
                    for (int q = 0; q < YP; ++q) *(bf16x4 *)&sm.m[q][m_at(t, s0)] = w[q];
                };
                // below the diagonal exp(S_t - S_s) is exp(S_t - S_e) exp(S_e - S_s), e the last token of the column's block
                auto below = [&](int tb, int sb, f32x4 v) {
                    const int t = 16 * tb + col, s0 = 16 * sb + 4 * g, end = 16 * sb + 15;
                    const float u = __builtin_amdgcn_exp2f((sm.sh[t] - sm.sh[end]) + (sm.sl[t] - sm.sl[end]));
                    put_block(t, s0, v * (*(const f32x4 *)&sm.block[s0] * u));
                };
                if (has0) g0 = block(tb0, tb0, g0);
                if (has1) g1 = block(tb1, sb1, g1);
                if (has2) g2 = block(tb2, sb2, g2);
                if (has0) {
                    const int t = 16 * tb0 + col, s0 = 16 * tb0 + 4 * g;
                    const f32x4 sh = *(const f32x4 *)&sm.sh[s0], sl = *(const f32x4 *)&sm.sl[s0], dl = *(const f32x4 *)&sm.delta[s0];
                    const float th = sm.sh[t], tl = sm.sl[t];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        g0[j] *= __builtin_amdgcn_exp2f((th - sh[j]) + (tl - sl[j])) * dl[j];
                        g0[j] = 4 * g + j > col ? 0.0f : 4 * g + j == col ? g0[j] + skip : g0[j];
                    }
                    put_block(t, s0, g0);
                }
                if (has1) below(tb1, sb1, g1);
                if (has2) below(tb2, sb2, g2);
                fetch_rows(rc, cp, a.c_stride, cs, next);
                // exp(S) C h0: rows p, column t in the lane
#pragma unroll
                for (int i = 0; i < QB; ++i) acc[i] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int n = 0; n < NPAD / 32; ++n) {
                    bf16x8 fh[YP], fc[QB][NP];
                    split(__builtin_shufflevector(h[2 * n], h[2 * n + 1], 0, 1, 2, 3, 4, 5, 6, 7), fh);
#pragma unroll
                    for (int i = 0; i < QB; ++i) {
                        const int at = at_c ^ 32 * n;
#pragma unroll
                        for (int q = 0; q < NP; ++q) {
                            const bf16 *const rows = &sm.c[q][16 * i * NPAD];
                            const bf16x4 lo = *(const bf16x4 *)(rows + at), hi = *(const bf16x4 *)(rows + (at ^ 16));
                            fc[i][q] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                        }
                    }
                    each_pair<YP, YP, NP>([&](int u, int v) {
#pragma unroll
                        for (int i = 0; i < QB; ++i) acc[i] = mma(fh[u], fc[i][v], acc[i]);
                    });
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int i = 0; i < QB; ++i) acc[i] *= __builtin_amdgcn_exp2f(sm.sh[16 * i + col]);
                __syncthreads();
            }
            fetch_x(next);
            Piece<T, 4> rz[FULL ? QB : 1];
            const int p4 = p_base + wave * 16 + 4 * g;       // rows of y that this lane stores
            const uint32_t out4 = p4 < P ? 0 : kOutside;
            if constexpr (FULL) {
                const Rows zrows = rows_at(a.z + (int64_t)(first + t0) * a.z_stride + hp, a.z ? left : 0, zs);
#pragma unroll
                for (int i = 0; i < QB; ++i)
                    rz[i].template load<WIDE>(zrows, (col * zs + p4 * e | out4) + 16 * i * zs, p4 < P ? P - p4 : 0);
            }

            bf16x8 fx[QK][NP];
#pragma unroll
            for (int k = 0; k < QK; ++k)
#pragma unroll
                for (int q = 0; q < NP; ++q) {
                    const bf16x4 lo = read_transposed(&sm.x[q][32 * k * 64 + at_x]);
                    const bf16x4 hi = read_transposed(&sm.x[q][(32 * k + 4) * 64 + (at_x ^ 8)]);
                    fx[k][q] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                }
            // the state behind the chunk
#pragma unroll
            for (int i = 0; i < NB; ++i) h[i] *= keep;
#pragma unroll
            for (int k = 0; k < QK; ++k) {
                const f32x4 w0 = *(const f32x4 *)&sm.into[32 * k + 8 * g], w1 = *(const f32x4 *)&sm.into[32 * k + 8 * g + 4];
                f32x8 x = __builtin_convertvector(fx[k][NP - 1], f32x8);
#pragma unroll
                for (int q = NP - 2; q >= 0; --q) x += __builtin_convertvector(fx[k][q], f32x8);
                bf16x8 fw[3];
                split(x * __builtin_shufflevector(w0, w1, 0, 1, 2, 3, 4, 5, 6, 7), fw);
                const int kStep = NB * NP <= 4 ? NB : NP == 1 ? 4 : 2;      // blocks of the state that go side by side
#pragma unroll
                for (int i0 = 0; i0 < NB; i0 += kStep) {
                    bf16x8 fb[kStep][NP];
#pragma unroll
                    for (int i = 0; i < kStep; ++i)
#pragma unroll
                        for (int q = 0; q < NP; ++q) {
                            const int at = at_b ^ 16 * (i0 + i);
                            const bf16x4 lo = read_transposed(&sm.b[q][32 * k * NPAD + at]);
                            const bf16x4 hi = read_transposed(&sm.b[q][(32 * k + 4) * NPAD + (at ^ 8)]);
                            fb[i][q] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                        }
                    each_pair<3, NP, 3>([&](int u, int v) {
#pragma unroll
                        for (int i = 0; i < kStep; ++i) h[i0 + i] = mma(fb[i][u], fw[v], h[i0 + i]);
                    });
                    __builtin_amdgcn_sched_barrier(0);       // (operands read further ahead do not fit the registers)
                }
            }

            if constexpr (FULL) {
#pragma unroll
                for (int k = 0; k < QK; ++k) {
                    bf16x8 fm[QB][YP];
#pragma unroll
                    for (int i = 2 * k; i < QB; ++i)
#pragma unroll
                        for (int q = 0; q < YP; ++q) fm[i][q] = *(const bf16x8 *)&sm.m[q][m_at(16 * i + col, 32 * k + 8 * g)];
                    each_pair<YP, NP, YP>([&](int u, int v) {
#pragma unroll
                        for (int i = 2 * k; i < QB; ++i) acc[i] = mma(fx[k][u], fm[i][v], acc[i]);
                    });
                }
                const Rows yrows = rows_at(a.y + (int64_t)(first + t0) * a.y_stride + hp, left, ys);
#pragma unroll
                for (int i = 0; i < QB; ++i) {
                    Piece<T, 4> out;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float v = acc[i][j];
                        odd = fmaf(v, 0.0f, odd);
                        if (a.z) v *= silu_as<T>((float)rz[i].v[j]);
                        out.v[j] = (T)v;
                    }
                    out.template store<WIDE>(yrows, (col * ys + p4 * e | out4) + 16 * i * ys, p4 < P ? P - p4 : 0);
                }
            }
            __syncthreads();
        }
        // An infinity or NaN among the operands, numbers beyond the largest bf16 one, sums that overflow: parts of an infinity do
        // not add up to it, and x of a token meets the zeros of M for the tokens before.  Any of it shows in y or in the state.
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) odd = fmaf(h[i][j], 0.0f, odd);
        const bool mine = __any(odd != 0.0f);
        if (lane == 0) sm.block[wave] = mine ? 1.0f : 0.0f;
        __syncthreads();
        const f32x4 any = *(const f32x4 *)&sm.block[0];
        if (__builtin_amdgcn_readfirstlane(any[0] + any[1] + any[2] + any[3] != 0.0f)) {
            const Again again = arguments_again();
            const Part v = locate(again, r);
            if (mine) get_before(again, v, h);
            walk(again, v, sm, mine, h);
        }
        if (!FULL) {
            put_state(&a, w.p, h, w.ws + (size_t)w.part * P * N, true);
            if (p_base == 0 && tid == 0) a.part_decay[w.ws_head * a.n_parts + w.part] = total;
        } else if (w.part == w.parts - 1) {
            put_state(&a, w.p, h, a.state_out + w.pool_at, a.state_out && w.slot >= 0);
        }
    }
};

// workgroups that share a compute unit, by LDS; rows that are moved element by element take more registers
template <typename Scan, bool WIDE> constexpr int scan_residents() { return sizeof(typename Scan::Shared) > 81920 ? 1 : sizeof(typename Scan::Shared) > 42000 || !WIDE ? 2 : 3; }

template <typename T, int NPAD, int Q, bool FULL, bool WIDE>
__global__ void __launch_bounds__(256, (scan_residents<SsmScan<T, NPAD, Q, FULL, WIDE>, WIDE>()))
ssm_scan_kernel(SsmArgs<T> a)
{
    typedef SsmScan<T, NPAD, Q, FULL, WIDE> Scan;
    __shared__ typename Scan::Shared sm;
    Scan::run(a, sm);
}

// What a part keeps of a number: an infinity stays one, also where the part's tokens together keep nothing in 32 bits.
__device__ inline float kept(float v, float decay) { return decay == 0.0f && fabsf(v) > 3.4028234e38f ? v : v * decay; }

// From what the parts' tokens leave to the states behind the parts: entry i of the workspace += decay of part i times entry
// i - 1, a lane to four numbers of a state.
template <typename T, int Q> __global__ void __launch_bounds__(256) ssm_join_kernel(SsmArgs<T> a)
{
    const int head = blockIdx.y, r = blockIdx.z;
    int first, length;
    request_rows(a.rq, r, &first, &length);
    const int parts = parts_of_request(a.part_chunks, a.n_parts, (length + Q - 1) / Q);
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
#pragma unroll
                for (int k = 0; k < 4; ++k) cur[k] = kept(cur[k], decay[i + j]) + e[j][k];
                *(f32x4 *)(ws + (i + j) * size) = cur;
            }
        }
    } else {
        for (int c = 0; c < 4 && at + c < size; ++c) {
            float cur = ws[c];
            for (int i = 1; i < parts - 1; ++i) ws[i * size + c] = cur = kept(cur, decay[i]) + ws[i * size + c];
        }
    }
}

}  // namespace wpk
#endif
