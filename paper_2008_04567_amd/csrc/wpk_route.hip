// The router of a layer of experts: every token's experts of the largest logits, their weights, and the order that sorts the
// tokens by expert.
//
// A token is taken by 16 lanes, or by a wave where there are more than 256 experts or 16 choices.  Lanes hold logits as integers of the
// same order, and k times the largest is found by maxima over lanes, of equal ones that of the lowest number, and taken away
// (bound: the instructions of these rounds).  The sorted order is a counting sort whose every step has one result: a chunk of
// tokens counts its experts, and the row of a token's choice is the expert's start, plus what earlier chunks, earlier waves of the
// chunk and earlier lanes chose.  Few tokens are one chunk and one launch; more are two (bound: launches and latencies).
#include "wpk_seq.h"

namespace wpk {

static const int kRouteThreads = 1024, kRouteWaves = kRouteThreads / 64, kMostExperts = 1024, kMostChosen = 32;
static const int kChunks = kComputeUnits;          // at most
static const int kOneChunk = 64;                   // tokens that are one

struct RouteArgs {
    const void *logits;
    int32_t *experts, *starts, *source, *place, *counts;
    float *weights;
    int32_t tokens, n, k, normalize, chunk, chunks;      // n experts; tokens of a chunk
    float scale;
    int64_t stride;
};

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
__host__ __device__ inline int counts_stride(int n) { return (n + 3) / 4 * 4; }      // between chunks

// ascending as the values are; zeros of both signs are one, NaN is -inf, and nothing is 0
__device__ inline uint32_t key_of(float v)
{
    if (v != v) v = -INFINITY;
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float value_of(uint32_t key)
{
    return __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// ... of a logit and its expert's number: the latter shares the integer where the former has 16 bits, lower numbers larger
template <typename T> struct Key {
    static __device__ uint32_t of(T v, int e)
    {
        const uint32_t b = __builtin_bit_cast(uint16_t, (T)value_of(key_of((float)v)));
        return ((b & 0x8000u ? ~b & 0xffffu : b | 0x8000u) << 16) | (uint32_t)(0xffff - e);
    }
    static __device__ int expert(uint32_t key) { return 0xffff - (int)(key & 0xffffu); }
    static __device__ float value(uint32_t key)
    {
        const uint32_t b = key >> 16;
        return (float)__builtin_bit_cast(T, (uint16_t)(b & 0x8000u ? b & 0x7fffu : ~b));
    }
};
template <> struct Key<float> {
    static __device__ uint32_t of(float v, int) { return key_of(v); }
    static __device__ float value(uint32_t key) { return value_of(key); }
};

template <int CTRL, int ROWS> __device__ inline uint32_t max_of_lane_before(uint32_t v)
{
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, true));
}
__device__ inline uint32_t wave_max(uint32_t v)
{
    v = max_of_lane_before<0x111, 0xf>(v);
    v = max_of_lane_before<0x112, 0xf>(v);
    v = max_of_lane_before<0x114, 0xf>(v);
    v = max_of_lane_before<0x118, 0xf>(v);
    v = max_of_lane_before<0x142, 0xa>(v);
    v = max_of_lane_before<0x143, 0xc>(v);
    return __builtin_amdgcn_readlane((int)v, 63);
}
// What follows the choice, in the lanes that have one: `key` is its, `top` the largest, `all` the sum of exp(logit - top) over all
// experts or, normalized, over the chosen.
__device__ inline void put_choice(const RouteArgs &a, int64_t at, int expert, float weight, float top, float all)
{
    a.experts[at] = expert;
    a.weights[at] = top == -INFINITY ? 0.0f : a.scale * (weight / all);
}

// One token's choice by a wave; lane j < k returns the j-th expert.  A lane holds neighbouring experts, so the lowest lane and its
// lowest entry win a tie.
template <typename T, int PER> __device__ inline int choose_by_wave(const RouteArgs &a, int token, int lane)
{
    const T *const row = (const T *)a.logits + (int64_t)token * a.stride;
    uint32_t key[PER];
    float v[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = lane * PER + i;
        key[i] = e < a.n ? key_of((float)row[min(e, a.n - 1)]) : 0;
        v[i] = value_of(key[i]);
    }
    int mine = 0;
    uint32_t mine_key = 0;
    for (int j = 0; j < a.k; ++j) {
        uint32_t best = key[0];
#pragma unroll
        for (int i = 1; i < PER; ++i) best = max(best, key[i]);
        const uint32_t most = wave_max(best);
        const int at = __builtin_ctzll(__ballot(best == most));
        int entry = 0;
#pragma unroll
        for (int i = PER - 1; i >= 0; --i)
            if (key[i] == most) entry = i;
        entry = __builtin_amdgcn_readlane(entry, at);
        if (lane == j) mine = at * PER + entry, mine_key = most;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (lane == at && i == entry) key[i] = 0;
    }
    const float top = value_of(__builtin_amdgcn_readlane((int)mine_key, 0));
    const float e = lane < a.k ? expf(value_of(mine_key) - top) : 0.0f;
    float sum = e;
    if (!a.normalize) {
        sum = 0.0f;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (lane * PER + i < a.n) sum += expf(v[i] - top);
    }
    sum = wave_total(sum);
    if (lane < a.k) put_choice(a, (int64_t)token * a.k + lane, mine, e, top, sum);
    return mine;
}

// ... of a row of 16 lanes, in all of them
template <int CTRL> __device__ inline uint32_t of_lane(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
__device__ inline uint32_t row_most(uint32_t v)
{
    v = max(v, of_lane<0xb1>(v));          // quad_perm 1 0 3 2
    v = max(v, of_lane<0x4e>(v));          // quad_perm 2 3 0 1
    v = max(v, of_lane<0x141>(v));         // row_half_mirror
    return max(v, of_lane<0x140>(v));      // row_mirror
}
__device__ inline float row_total(float v)
{
    v += __builtin_bit_cast(float, of_lane<0xb1>(__builtin_bit_cast(uint32_t, v)));
    v += __builtin_bit_cast(float, of_lane<0x4e>(__builtin_bit_cast(uint32_t, v)));
    v += __builtin_bit_cast(float, of_lane<0x141>(__builtin_bit_cast(uint32_t, v)));
    return v + __builtin_bit_cast(float, of_lane<0x140>(__builtin_bit_cast(uint32_t, v)));
}

// Four tokens' choices by a wave, 16 lanes each; lane j < k of a token returns its j-th expert, -1 of a token that is not there (which
// chooses as the last one).  Lane l holds experts l, l + 16 ..; a logit of 16 bits shares an integer with the expert's number, so
// that one maximum finds both, and of 32 bits a second one finds the lowest number among the equal.
template <typename T, int PER> __device__ inline int choose_by_row(const RouteArgs &a, int token, int end)
{
    const int lane = threadIdx.x & 15;
    const T *const row = (const T *)a.logits + (int64_t)min(token, end - 1) * a.stride;
    uint32_t key[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = 16 * i + lane;
        key[i] = e < a.n ? Key<T>::of(row[min(e, a.n - 1)], e) : 0;
    }
    uint32_t mine_key = 0, mine = 0;
    for (int j = 0; j < a.k; ++j) {
        uint32_t most = key[0];
#pragma unroll
        for (int i = 1; i < PER; ++i) most = max(most, key[i]);
        most = row_most(most);
        if constexpr (sizeof(T) == 2) {
            if (lane == j) mine_key = most;
#pragma unroll
            for (int i = 0; i < PER; ++i) key[i] = key[i] == most ? 0 : key[i];
        } else {
            uint32_t left = 0;                                 // 1024 less the number
#pragma unroll
            for (int i = PER - 1; i >= 0; --i) left = key[i] == most ? 1024 - (16 * i + lane) : left;
            left = row_most(left);
            if (lane == j) mine_key = most, mine = 1024 - left;
#pragma unroll
            for (int i = 0; i < PER; ++i) key[i] = 1024 - (16 * i + lane) == left ? 0 : key[i];
        }
    }
    if constexpr (sizeof(T) == 2) mine = Key<T>::expert(mine_key);
    const float mine_v = Key<T>::value(mine_key), top = __shfl(mine_v, 0, 16);
    const float e = lane < a.k ? expf(mine_v - top) : 0.0f;
    float sum = e;
    if (!a.normalize) {
        sum = 0.0f;
        for (int i = 0; i < PER; ++i)
            if (16 * i + lane < a.n) sum += expf(value_of(key_of((float)row[16 * i + lane])) - top);
    }
    sum = row_total(sum);
    if (token >= end) return -1;
    if (lane < a.k) put_choice(a, (int64_t)token * a.k + lane, mine, e, top, sum);
    return mine;
}

// Exclusive sums over the experts, one a thread, of all threads.
__device__ inline int sum_before(int v, int *room)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int upto = running_sum_32(v);
    if (lane == 63) room[wave] = upto;
    __syncthreads();
    int before = upto - v;
#pragma unroll
    for (int w = 0; w < kRouteWaves; ++w)
        if (w < wave) before += room[w];
    __syncthreads();
    return before;
}

// The waves take equal runs of a chunk's choices, `ids` (the chunk's first at 0), count them, and number them in order: a choice's
// row is the expert's first row for the chunk, plus what earlier waves and earlier lanes chose.  counts: room for a row of experts a
// wave, zeros.
struct Runs {
    int waves, run;                   // waves that have one; choices of a run
    __device__ Runs(const RouteArgs &a, int choices)
    {
        const int most = min(min(kRouteWaves, 8 * kMostExperts / a.n), (choices + 63) / 64);
        run = ((choices + most - 1) / most + 63) / 64 * 64;
        waves = (choices + run - 1) / run;
    }
};
__device__ inline void count_runs(const RouteArgs &a, const Runs &r, const int32_t *ids, int choices, int *counts)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (wave >= r.waves) return;
    const int end = min((wave + 1) * r.run, choices);
    for (int f = wave * r.run + lane; f < end; f += 64) atomicAdd(&counts[wave * a.n + ids[f]], 1);
}
// the counts of expert e become the rows before the waves' choices, from `at` on; returns the row behind them
__device__ inline int rows_of_runs(const RouteArgs &a, const Runs &r, int *counts, int e, int at)
{
    for (int w = 0; w < r.waves; ++w) {
        const int c = counts[w * a.n + e];
        counts[w * a.n + e] = at;
        at += c;
    }
    return at;
}
__device__ inline void place_runs(const RouteArgs &a, const Runs &r, const int32_t *ids, int choices, int64_t f0, int *counts)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (wave >= r.waves) return;
    int *const row = counts + wave * a.n;
    const int end = min((wave + 1) * r.run, choices);
    const uint64_t before = (1ull << lane) - 1;
    for (int f = wave * r.run; f < end; f += 64) {
        const bool there = f + lane < end;
        const int e = there ? ids[f + lane] : 0;
        uint64_t same = __ballot(there);                       // lanes that chose the same expert
        for (int b = 1; b < a.n; b *= 2) {
            const uint64_t set = __ballot((e & b) != 0);
            same &= (e & b) ? set : ~set;
        }
        const int at = row[e];
        if (there) {
            const int to = at + __popcll(same & before);
            a.place[f0 + f + lane] = to;
            a.source[to] = (int)((f0 + f + lane) / a.k);
            if ((same & before) == 0) row[e] = at + __popcll(same);
        }
    }
}

// A workgroup chooses for a chunk of tokens, and counts its experts; the only chunk is put in order as well.  32 tokens of 64 experts,
// eight chosen, fp32: 5.3 us, all of it; 16384 tokens of 128, bf16: 7.1 us and 6.7 for the order (a wave a token took 12.4).
template <typename T, int PER, bool ROW> __global__ void __launch_bounds__(kRouteThreads) route_choose_kernel(RouteArgs a)
{
    __shared__ int counts[8 * kMostExperts], room[kRouteWaves], ids[kOneChunk * kMostChosen];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int t0 = blockIdx.x * a.chunk, t1 = min(t0 + a.chunk, a.tokens), choices = (t1 - t0) * a.k;
    const bool order = a.starts != nullptr, only = a.chunks == 1;
    const Runs runs(a, choices);
    if (order)
        for (int i = tid; i < (only ? runs.waves : 1) * a.n; i += kRouteThreads) counts[i] = 0;
    __syncthreads();
    const int kTokens = ROW ? 4 : 1, kSlots = ROW ? 16 : 64, j = lane % kSlots;
    for (int t = t0 + wave * kTokens; t < t1; t += kRouteWaves * kTokens) {
        const int token = t + lane / kSlots;
        int e;
        if constexpr (ROW) e = choose_by_row<T, PER>(a, token, t1);
        else e = choose_by_wave<T, PER>(a, token, lane);
        if (order && j < a.k && e >= 0) {
            if (only) ids[(token - t0) * a.k + j] = e;
            else atomicAdd(&counts[e], 1);
        }
    }
    if (!order) return;
    __syncthreads();
    if (!only) {
        if (tid < counts_stride(a.n)) a.counts[(int64_t)blockIdx.x * counts_stride(a.n) + tid] = tid < a.n ? counts[tid] : 0;
        return;
    }
    count_runs(a, runs, ids, choices, counts);
    __syncthreads();
    const int mine = tid < a.n ? rows_of_runs(a, runs, counts, tid, 0) : 0, start = sum_before(mine, room);
    if (tid < a.n) {
        for (int w = 0; w < runs.waves; ++w) counts[w * a.n + tid] += start;
        a.starts[tid] = start;
        if (tid == a.n - 1) a.starts[a.n] = start + mine;
    }
    __syncthreads();
    place_runs(a, runs, ids, choices, 0, counts);
}

// Every workgroup adds up all chunks' counts for itself (128 KiB from the caches at 256 chunks of 128 experts): a launch less than a
// kernel between, which would take as long as the sums do.
__global__ void __launch_bounds__(kRouteThreads) route_place_kernel(RouteArgs a)
{
    __shared__ int total[kMostExperts], base[kMostExperts], counts[8 * kMostExperts], room[kRouteWaves];
    const int tid = threadIdx.x, chunk = blockIdx.x;
    const int64_t f0 = (int64_t)chunk * a.chunk * a.k;
    const int choices = (min(chunk * a.chunk + a.chunk, a.tokens) - chunk * a.chunk) * a.k;
    const int32_t *const ids = a.experts + f0;
    const Runs runs(a, choices);
    if (tid < a.n) total[tid] = base[tid] = 0;
    for (int i = tid; i < runs.waves * a.n; i += kRouteThreads) counts[i] = 0;
    __syncthreads();
    // four experts a thread, as many chunks at once as there are threads for
    const int stride = counts_stride(a.n);
    int wide = 1;
    while (4 * wide < a.n) wide *= 2;
    const int e = 4 * (tid % wide), part = tid / wide, parts = kRouteThreads / wide;
    if (e < a.n) {
        i32x4 all = {0, 0, 0, 0}, earlier = {0, 0, 0, 0};
#pragma unroll 8
        for (int c = part; c < a.chunks; c += parts) {
            const i32x4 v = *(const i32x4 *)(a.counts + (int64_t)c * stride + e);
            all += v;
            if (c < chunk) earlier += v;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (e + i >= a.n) continue;
            atomicAdd(&total[e + i], all[i]);
            atomicAdd(&base[e + i], earlier[i]);
        }
    }
    count_runs(a, runs, ids, choices, counts);
    __syncthreads();
    const int mine = tid < a.n ? total[tid] : 0, start = sum_before(mine, room);
    if (tid < a.n) {
        rows_of_runs(a, runs, counts, tid, start + base[tid]);
        if (chunk == 0) {
            a.starts[tid] = start;
            if (tid == a.n - 1) a.starts[a.n] = start + mine;
        }
    }
    __syncthreads();
    place_runs(a, runs, ids, choices, f0, counts);
}

__global__ void route_nothing_kernel(int32_t *starts, int32_t n)      // no tokens: every expert has none
{
    for (int i = threadIdx.x; i <= n; i += blockDim.x) starts[i] = 0;
}

static int chunk_tokens(int tokens)
{
    const int each = (tokens + kChunks - 1) / kChunks;
    return each > kOneChunk ? each : kOneChunk;            // (as many as a workgroup takes at once)
}

static int check_route(const wpk_route_desc *dp)
{
    if (!dp) return WPK_E_NULL_PTR;
    const wpk_route_desc &d = *dp;
    if (d.tokens < 0 || d.experts < 1 || d.k < 1 || d.k > d.experts || d.logits_stride < d.experts) return WPK_E_BAD_DESC;
    if (d.experts > kMostExperts || d.k > kMostChosen || !seq_type_ok(d.dtype) || (int64_t)d.tokens * d.k > kMostRows ||
        d.logits_stride >= 1ll << 30 || (d.normalize != 0 && d.normalize != 1))
        return WPK_E_UNSUPPORTED;
    return WPK_OK;
}

template <typename T> static int route_typed(const RouteArgs &a, hipStream_t st)
{
    const dim3 grid(a.chunks), block(kRouteThreads);
    const bool row = a.k <= 16;
    if (row && a.n <= 32) hipLaunchKernelGGL((route_choose_kernel<T, 2, true>), grid, block, 0, st, a);
    else if (row && a.n <= 64) hipLaunchKernelGGL((route_choose_kernel<T, 4, true>), grid, block, 0, st, a);
    else if (row && a.n <= 128) hipLaunchKernelGGL((route_choose_kernel<T, 8, true>), grid, block, 0, st, a);
    else if (row && a.n <= 256) hipLaunchKernelGGL((route_choose_kernel<T, 16, true>), grid, block, 0, st, a);
    else if (a.n <= 256) hipLaunchKernelGGL((route_choose_kernel<T, 4, false>), grid, block, 0, st, a);
    else if (a.n <= 512) hipLaunchKernelGGL((route_choose_kernel<T, 8, false>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((route_choose_kernel<T, 16, false>), grid, block, 0, st, a);
    WPK_HIP(hipGetLastError());
    if (!a.starts || a.chunks == 1) return WPK_OK;
    hipLaunchKernelGGL(route_place_kernel, grid, block, 0, st, a);
    WPK_HIP(hipGetLastError());
    return WPK_OK;
}

}  // namespace wpk

extern "C" {

int64_t wpk_route_workspace_bytes(const wpk_route_desc *d)
{
    const int rc = wpk::check_route(d);
    if (rc != WPK_OK) return rc;
    const int64_t chunk = wpk::chunk_tokens(d->tokens), chunks = (d->tokens + chunk - 1) / chunk;
    return chunks < 2 ? 0 : chunks * wpk::counts_stride(d->experts) * (int64_t)sizeof(int32_t);
}

int wpk_route_fwd(const wpk_route_desc *dp, const void *logits, int32_t *experts, float *weights, int32_t *starts,
                  int32_t *source, int32_t *place, void *workspace, void *stream)
{
    using namespace wpk;
    const int rc = check_route(dp);
    if (rc != WPK_OK) return rc;
    const wpk_route_desc d = *dp;
    const bool order = starts || source || place;
    if (order && (!starts || (d.tokens > 0 && (!source || !place)))) return WPK_E_NULL_PTR;
    if (!aligned_to(starts, 4) || !aligned_to(source, 4) || !aligned_to(place, 4) || !aligned_to(experts, 4) || !aligned_to(weights, 4) ||
        !aligned_to(logits, seq_type_bytes(d.dtype)) || !aligned_to(workspace, 16))
        return WPK_E_BAD_ARG;
    const hipStream_t st = (hipStream_t)stream;
    if (d.tokens == 0) {
        if (order) {
            hipLaunchKernelGGL(route_nothing_kernel, dim3(1), dim3(256), 0, st, starts, d.experts);
            WPK_HIP(hipGetLastError());
        }
        return WPK_OK;
    }
    if (!logits || !experts || !weights) return WPK_E_NULL_PTR;
    const int chunk = chunk_tokens(d.tokens), chunks = (d.tokens + chunk - 1) / chunk;
    if (order && chunks > 1 && !workspace) return WPK_E_NULL_PTR;
    const RouteArgs a = {logits, experts, starts, source, place, (int32_t *)workspace, weights, d.tokens, d.experts, d.k, d.normalize,
                         chunk, chunks, d.scale, d.logits_stride};
    if (d.dtype == WPK_BF16) return route_typed<bf16>(a, st);
    if (d.dtype == WPK_F16) return route_typed<f16>(a, st);
    return route_typed<float>(a, st);
}

}  // extern "C"
