// The router of a layer of experts: every token's experts of the largest logits, their weights, and the order that sorts the
// tokens by expert.
//
// A wave takes a token: a lane holds neighbouring experts' logits as integers of the same order, and k times the largest is found
// by sums (maxima) over lanes and taken away; the lowest lane and the lowest entry win a tie.  The sorted order is a counting sort
// whose every step has one result: a chunk of tokens counts its experts, and the row of a token's choice is the expert's start,
// plus what earlier chunks, earlier waves of the chunk and earlier lanes chose.  Few tokens are one chunk and one launch; more are
// two (bound: launches and latencies).
#include "wpk_seq.h"

namespace wpk {

static const int kRouteThreads = 1024, kRouteWaves = kRouteThreads / 64, kMostExperts = 1024;
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
__device__ inline float wave_total(float v)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    return v;
}

// One token's choice; lane j < k returns the j-th expert, and its weight is stored.
template <typename T, int PER> __device__ inline int choose(const RouteArgs &a, int token, int lane)
{
    const T *const row = (const T *)a.logits + (int64_t)token * a.stride;
    uint32_t key[PER];
    float v[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = lane * PER + i;
        const float t = e < a.n ? (float)row[e] : 0.0f;
        key[i] = e < a.n ? key_of(t) : 0;
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
    if (lane < a.k) {
        a.experts[(int64_t)token * a.k + lane] = mine;
        a.weights[(int64_t)token * a.k + lane] = top == -INFINITY ? 0.0f : a.scale * (e / sum);
    }
    return mine;
}

// Exclusive sums over the experts, one a thread, of all threads.
__device__ inline int sum_before(int v, int *room)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int upto = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 63) room[wave] = upto;
    __syncthreads();
    int before = upto - v;
#pragma unroll
    for (int w = 0; w < kRouteWaves; ++w)
        if (w < wave) before += room[w];
    __syncthreads();
    return before;
}

// Rows of the choices of a chunk's tokens [t0, t1): base[e] is the row of the chunk's first choice of expert e.  The waves take
// equal runs of the choices, count them, and number them in order.  counts: room for a row of experts a wave.
__device__ inline void place_chunk(const RouteArgs &a, int t0, int t1, const int *base, int *counts)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int waves = min(kRouteWaves, 8 * kMostExperts / a.n);
    const int64_t f0 = (int64_t)t0 * a.k, f1 = (int64_t)t1 * a.k;
    const int64_t run = ((f1 - f0 + waves - 1) / waves + 63) / 64 * 64;
    const int64_t begin = min(f0 + run * wave, f1), end = min(begin + run, f1);
    int *const row = counts + min(wave, waves - 1) * a.n;
    for (int i = threadIdx.x; i < waves * a.n; i += kRouteThreads) counts[i] = 0;
    __syncthreads();
    if (wave < waves)
        for (int64_t f = begin + lane; f < end; f += 64) atomicAdd(&row[a.experts[f]], 1);
    __syncthreads();
    for (int e = threadIdx.x; e < a.n; e += kRouteThreads) {
        int at = base[e];
        for (int w = 0; w < waves; ++w) {
            const int c = counts[w * a.n + e];
            counts[w * a.n + e] = at;
            at += c;
        }
    }
    __syncthreads();
    if (wave >= waves) return;
    const uint64_t before = (1ull << lane) - 1;
    for (int64_t f = begin; f < end; f += 64) {
        const bool there = f + lane < end;
        const int e = there ? a.experts[f + lane] : 0;
        uint64_t same = __ballot(there);                       // lanes that chose the same expert
        for (int b = 1; b < a.n; b *= 2) {
            const uint64_t set = __ballot((e & b) != 0);
            same &= (e & b) ? set : ~set;
        }
        const int at = row[e];
        if (there) {
            const int r = at + __popcll(same & before);
            a.place[f + lane] = r;
            a.source[r] = (int)((f + lane) / a.k);
            if ((same & before) == 0) row[e] = at + __popcll(same);
        }
    }
}

// A workgroup chooses for a chunk of tokens, and counts its experts; the only chunk is put in order as well.
template <typename T, int PER> __global__ void __launch_bounds__(kRouteThreads) route_choose_kernel(RouteArgs a)
{
    __shared__ int hist[kMostExperts], counts[8 * kMostExperts], room[kRouteWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int t0 = blockIdx.x * a.chunk, t1 = min(t0 + a.chunk, a.tokens);
    if (tid < a.n) hist[tid] = 0;
    __syncthreads();
    for (int t = t0 + wave; t < t1; t += kRouteWaves) {
        const int e = choose<T, PER>(a, t, lane);
        if (lane < a.k && a.starts) atomicAdd(&hist[e], 1);
    }
    if (!a.starts) return;
    __syncthreads();
    const int mine = tid < a.n ? hist[tid] : 0;
    if (a.chunks > 1) {
        if (tid < a.n) a.counts[(int64_t)blockIdx.x * a.n + tid] = mine;
        return;
    }
    const int start = sum_before(mine, room);
    if (tid < a.n) {
        hist[tid] = start;
        a.starts[tid] = start;
        if (tid == a.n - 1) a.starts[a.n] = start + mine;
    }
    __syncthreads();
    place_chunk(a, t0, t1, hist, counts);
}

__global__ void __launch_bounds__(kRouteThreads) route_place_kernel(RouteArgs a)
{
    __shared__ int total[kMostExperts], base[kMostExperts], counts[8 * kMostExperts], room[kRouteWaves];
    const int tid = threadIdx.x, chunk = blockIdx.x;
    if (tid < a.n) total[tid] = base[tid] = 0;
    __syncthreads();
    int wide = 1;
    while (wide < a.n) wide *= 2;
    const int e = tid % wide, part = tid / wide, parts = kRouteThreads / wide;
    if (e < a.n) {
        int all = 0, earlier = 0;
#pragma unroll 8
        for (int c = part; c < a.chunks; c += parts) {
            const int v = a.counts[(int64_t)c * a.n + e];
            all += v;
            if (c < chunk) earlier += v;
        }
        atomicAdd(&total[e], all);
        atomicAdd(&base[e], earlier);
    }
    __syncthreads();
    const int mine = tid < a.n ? total[tid] : 0, start = sum_before(mine, room);
    if (tid < a.n) {
        base[tid] += start;
        if (chunk == 0) {
            a.starts[tid] = start;
            if (tid == a.n - 1) a.starts[a.n] = start + mine;
        }
    }
    __syncthreads();
    place_chunk(a, chunk * a.chunk, min(chunk * a.chunk + a.chunk, a.tokens), base, counts);
}

__global__ void route_nothing_kernel(int32_t *starts, int32_t n)      // no tokens: every expert has none
{
    for (int i = threadIdx.x; i <= n; i += blockDim.x) starts[i] = 0;
}

static int chunk_tokens(int tokens)
{
    return tokens <= kOneChunk ? kOneChunk : (tokens + kChunks - 1) / kChunks > 16 ? (tokens + kChunks - 1) / kChunks : 16;
}

static int check_route(const wpk_route_desc *dp)
{
    if (!dp) return WPK_E_NULL_PTR;
    const wpk_route_desc &d = *dp;
    if (d.tokens < 0 || d.experts < 1 || d.k < 1 || d.k > d.experts || d.logits_stride < d.experts) return WPK_E_BAD_DESC;
    if (d.experts > kMostExperts || d.k > 32 || !seq_type_ok(d.dtype) || (int64_t)d.tokens * d.k > kMostRows ||
        d.logits_stride >= 1ll << 30 || (d.normalize != 0 && d.normalize != 1))
        return WPK_E_UNSUPPORTED;
    return WPK_OK;
}

template <typename T> static int route_typed(const RouteArgs &a, hipStream_t st)
{
    const dim3 grid(a.chunks), block(kRouteThreads);
    if (a.n <= 64) hipLaunchKernelGGL((route_choose_kernel<T, 1>), grid, block, 0, st, a);
    else if (a.n <= 128) hipLaunchKernelGGL((route_choose_kernel<T, 2>), grid, block, 0, st, a);
    else if (a.n <= 256) hipLaunchKernelGGL((route_choose_kernel<T, 4>), grid, block, 0, st, a);
    else if (a.n <= 512) hipLaunchKernelGGL((route_choose_kernel<T, 8>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((route_choose_kernel<T, 16>), grid, block, 0, st, a);
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
    return chunks < 2 ? 0 : chunks * d->experts * (int64_t)sizeof(int32_t);
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
