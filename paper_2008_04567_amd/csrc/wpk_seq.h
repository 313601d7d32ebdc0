// What the sequence layers' translation units share: element types, activations, requests and their states.
#ifndef WPK_SEQ_H
#define WPK_SEQ_H

#include <hip/hip_runtime.h>
#include <math.h>

#include "wpk_internal.h"

#define WPK_HIP(call)                                  \
    do {                                               \
        hipError_t e_ = (call);                        \
        if (e_ != hipSuccess) {                        \
            set_last_hip_error((int)e_);               \
            return WPK_E_HIP;                          \
        }                                              \
    } while (0)

namespace wpk {

typedef __bf16 bf16;
typedef _Float16 f16;
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

static const int kComputeUnits = 256;   // of an MI355X: what launches are shaped for

inline int seq_type_bytes(int dtype) { return dtype == WPK_F32 ? 4 : 2; }
inline bool seq_type_ok(int dtype) { return dtype == WPK_F32 || dtype == WPK_BF16 || dtype == WPK_F16; }
inline bool aligned_to(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// exp and log of 32-bit results: within two units of the last place over the whole range
__device__ inline float silu(float v) { return v / (1.0f + expf(-v)); }
// The same on the reciprocal and exponential units, for values rounded to 16 bits next.  Relative error (2 |v| + 8) 2^-24, the
// first term from the exponent's rounding: 2^-21 for small |v|, 2^-19 at -10, 2^-17 at -60.  Below -88 the result is zero.
__device__ inline float silu_fast(float v)
{
    return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * v));
}
template <typename T> __device__ inline float silu_as(float v) { return sizeof(T) == 4 ? silu(v) : silu_fast(v); }
__device__ inline float softplus(float v) { return fmaxf(v, 0.0f) + log1pf(expf(-fabsf(v))); }

// log(1 + e) as log(u) e / (u - 1) with u = 1 + e rounded (Goldberg 1991, theorem 4): the quotient makes up for what the
// rounding lost, so the result is good to some ten units of 2^-24 however small e is.  e = exp(-|v|) is as good for all v: what
// the product with log2(e) loses, |v| 2^-24 of e, is put back (the rest of the product, and of log2(e), to first order).
__device__ inline float softplus_fast(float v)
{
    const float n = -fabsf(v), p = 1.44269502f * n, rest = fmaf(1.92596303e-8f, n, fmaf(1.44269502f, n, -p));
    const float e0 = __builtin_amdgcn_exp2f(p), e = n < -128.0f ? 0.0f : fmaf(e0, 0.693147182f * rest, e0);   // (NaN stays)
    const float u = 1.0f + e, d = u - 1.0f;
    const float l = d == 0.0f ? e : 0.69314718f * __builtin_amdgcn_logf(u) * (e * __builtin_amdgcn_rcpf(d));
    return fmaxf(v, 0.0f) + l;
}

// ---- sums over the lanes before, in 64 bits: data moves within rows of 16 lanes and then from row ends on -----------
template <int CTRL, int ROWS> __device__ inline double lanes_before(double v)      // zero where there is none
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROWS, 0xf, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, ROWS, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ inline double running_sum(double v)
{
    v += lanes_before<0x111, 0xf>(v);     // row_shr 1, 2, 4, 8
    v += lanes_before<0x112, 0xf>(v);
    v += lanes_before<0x114, 0xf>(v);
    v += lanes_before<0x118, 0xf>(v);
    v += lanes_before<0x142, 0xa>(v);     // lane 15 of a row to the next row: into rows 1 and 3
    v += lanes_before<0x143, 0xc>(v);     // lane 31 to the next two rows: into rows 2 and 3
    return v;
}

__device__ inline double read_lane(double v, int lane)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, lane), hi = __builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// what the last lane of a lane's row of 16 holds
__device__ inline double row_end(double v)
{
    const double e0 = read_lane(v, 15), e1 = read_lane(v, 31), e2 = read_lane(v, 47), e3 = read_lane(v, 63);
    const int row = (threadIdx.x >> 4) & 3;
    return row < 2 ? (row == 0 ? e0 : e1) : (row == 2 ? e2 : e3);
}

// v (1 + erf(v / sqrt 2)) / 2, below zero as v erfc(-v / sqrt 2) / 2: 1 + erf would cancel
__device__ inline float gelu(float v) { return 0.5f * v * erfcf(-0.70710678f * v); }
// The same for values rounded to 16 bits next.  erfc(x) / 2 is taken as t P(t) exp(-x^2), t = 1 / (1 + 0.44 x), with P of degree
// five fitted to the least largest relative error, 5.2e-6 for x up to 9.4 (beyond, erfc is no 32-bit number); the exponent's
// roundings add v^2 2^-23.
__device__ inline float gelu_fast(float v)
{
    const float a = fabsf(v), t = __builtin_amdgcn_rcpf(fmaf(0.311126984f, a, 1.0f));
    float s = fmaf(t, -0.0730525404f, 0.175324917f);
    s = fmaf(t, s, 0.020367641f);
    s = fmaf(t, s, 0.131791681f);
    s = fmaf(t, s, 0.12128526f);
    s = fmaf(t, s, 0.124280453f);
    s = t * s * __builtin_amdgcn_exp2f(-0.72134752f * a * a);
    return v * (v < 0.0f ? s : 1.0f - s);
}
template <typename T> __device__ inline float gelu_as(float v) { return sizeof(T) == 4 ? gelu(v) : gelu_fast(v); }

// the activation of four values; T: what they are rounded to next
template <typename T> __device__ inline f32x4 apply_act(f32x4 v, int act)
{
    if (act == WPK_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = v[i] < 0.0f ? 0.0f : v[i];         // (NaN stays)
    } else if (act == WPK_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = silu_as<T>(v[i]);
    } else if (act == WPK_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = gelu_as<T>(v[i]);
    }
    return v;
}

// ---- rows through buffer descriptors: what is outside a tensor reads as zero and is not written, without a branch -----
typedef __amdgpu_buffer_rsrc_t Rows;
static const uint32_t kOutside = 0x80000000u;    // an offset that no descriptor reaches, nor with a tile's rows added
// `rows` rows (none where that is negative) of `stride` bytes, together below 2^31
__device__ inline Rows rows_at(const void *base, int rows, uint32_t stride)
{
    return __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, __builtin_amdgcn_readfirstlane(max(rows, 0)) * stride, 0x00020000);
}

// V elements of a row from `offset` on, of which `left` are there.  Rows that are aligned are moved at once: all V are there
// or, with an offset that is outside, none.
template <typename T, int V> struct Piece {
    static const int words = V * (int)sizeof(T) / 4;
    typedef T vec_t __attribute__((ext_vector_type(V)));
    vec_t v;

    template <bool WIDE> __device__ void load(Rows rows, uint32_t offset, int left)
    {
        if constexpr (WIDE && words == 2) {
            v = __builtin_bit_cast(vec_t, __builtin_amdgcn_raw_buffer_load_b64(rows, offset, 0, 0));
        } else if constexpr (WIDE && words == 4) {
            v = __builtin_bit_cast(vec_t, __builtin_amdgcn_raw_buffer_load_b128(rows, offset, 0, 0));
        } else if constexpr (WIDE) {
            struct {
                u32x4 q[words / 4];
            } u;
#pragma unroll
            for (int i = 0; i < words / 4; ++i) u.q[i] = __builtin_amdgcn_raw_buffer_load_b128(rows, offset + 16 * i, 0, 0);
            v = __builtin_bit_cast(vec_t, u);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t at = i < left ? offset + i * (uint32_t)sizeof(T) : kOutside;
                if constexpr (sizeof(T) == 2) v[i] = __builtin_bit_cast(T, (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rows, at, 0, 0));
                else v[i] = __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b32(rows, at, 0, 0));
            }
        }
    }

    template <bool WIDE> __device__ void store(Rows rows, uint32_t offset, int left) const
    {
        if constexpr (WIDE && words == 2) {
            __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), rows, offset, 0, 0);
        } else if constexpr (WIDE && words == 4) {
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), rows, offset, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t at = i < left ? offset + i * (uint32_t)sizeof(T) : kOutside;
                if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, (T)v[i]), rows, at, 0, 0);
                else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, (T)v[i]), rows, at, 0, 0);
            }
        }
    }
};

// 16 bytes a lane from `rows` at the lane's `offset` plus `step` straight to LDS, one lane's behind the other's from `lds`
// on.  Not counted by the compiler: wait with s_waitcnt vmcnt before a barrier that lets anyone read them.
__device__ inline uint32_t lds_offset(const void *p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)p; }
__device__ inline void load_to_lds(Rows rows, uint32_t offset, uint32_t step, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %2\n s_nop 0\n buffer_load_dwordx4 %0, %1, %3 offen lds"
                 :
                 : "v"(offset), "s"(rows), "s"(lds), "s"(step)
                 : "m0", "memory");
}

// ---- requests and their states (wpk.h, "sequence layers") ------------------------------------------------
struct Requests {
    const int32_t *starts, *slot_map, *resume;
    int32_t tokens, max_length, slots;
};

// rows [first, first + length) of request i, the same for all lanes as i is (and known to be)
__device__ inline void request_rows(const Requests &q, int i, int *first, int *length)
{
    if (q.starts) {
        const int a = min(max(q.starts[i], 0), q.tokens), b = min(max(q.starts[i + 1], 0), q.tokens);
        *first = __builtin_amdgcn_readfirstlane(a);
        *length = __builtin_amdgcn_readfirstlane(max(b - a, 0));
    } else {
        *first = i * q.max_length;
        *length = q.max_length;
    }
}

// entry of request i's state, or -1
__device__ inline int request_slot(const Requests &q, int i)
{
    const int s = q.slot_map ? __builtin_amdgcn_readfirstlane(q.slot_map[i]) : i;
    return s >= 0 && s < q.slots ? s : -1;
}

__device__ inline bool request_resumes(const Requests &q, int i)
{
    return !q.resume || __builtin_amdgcn_readfirstlane(q.resume[i]) != 0;
}

static const int32_t kMostRows = 1 << 30;      // of any matrix: row numbers of whole tiles and chunks stay below 2^31

// tokens that the longest request can have, one at least: launches are shaped by max_length, which may be any upper bound
inline int32_t longest_request(int32_t tokens, int32_t max_length)
{
    return max_length < tokens ? max_length : tokens > 0 ? tokens : 1;
}

// What the two kinds of call check alike; `step` for the calls of one token a request.
inline int check_requests(int32_t sequences, int32_t tokens, int32_t max_length, int32_t slots, bool step, const void *starts,
                          const void *slot_map, const void *resume, const void *state_in, const void *state_out,
                          size_t state_align)
{
    if (step && (tokens != sequences || max_length != 1)) return WPK_E_BAD_ARG;
    if (!starts && (int64_t)sequences * max_length != tokens) return WPK_E_BAD_ARG;
    if ((state_in || state_out) && (slots < 1 || (!slot_map && slots < sequences))) return WPK_E_BAD_ARG;
    if (!aligned_to(starts, 4) || !aligned_to(slot_map, 4) || !aligned_to(resume, 4)) return WPK_E_BAD_ARG;
    if (!aligned_to(state_in, state_align) || !aligned_to(state_out, state_align)) return WPK_E_BAD_ARG;
    return WPK_OK;
}

}  // namespace wpk
#endif
