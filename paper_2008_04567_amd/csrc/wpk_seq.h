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
// the same on the reciprocal and exponential units (relative error about 2^-21): for values rounded to 16 bits next
__device__ inline float silu_fast(float v)
{
    return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * v));
}
template <typename T> __device__ inline float silu_as(float v) { return sizeof(T) == 4 ? silu(v) : silu_fast(v); }
__device__ inline float softplus(float v) { return fmaxf(v, 0.0f) + log1pf(expf(-fabsf(v))); }

template <typename T> __device__ inline float apply_act(float v, int act)
{
    if (act == WPK_ACT_RELU) return v < 0.0f ? 0.0f : v;                  // (NaN stays)
    if (act == WPK_ACT_SILU) return silu_as<T>(v);
    if (act == WPK_ACT_GELU) return 0.5f * v * (1.0f + erff(v * 0.70710678f));
    return v;
}

// ---- rows through buffer descriptors: what is outside a tensor reads as zero and is not written, without a branch -----
typedef __amdgpu_buffer_rsrc_t Rows;
static const uint32_t kOutside = 0x80000000u;    // an offset that no descriptor reaches
__device__ inline Rows rows_at(const void *base)
{
    return __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, 0x7fffffff, 0x00020000);
}

// V elements of a row, `left` of them there (none if the row is not): at once, or one by one where rows are not aligned
template <typename T, int V> struct Piece {
    static const int words = V * (int)sizeof(T) / 4;
    typedef T vec_t __attribute__((ext_vector_type(V)));
    vec_t v;

    // (`step`: bytes that are the same for all lanes)
    template <bool WIDE> __device__ void load(Rows rows, uint32_t offset, uint32_t step, int left)
    {
        if constexpr (WIDE) {
            const uint32_t at = left > 0 ? offset : kOutside;
            union {
                uint32_t w[words];
                vec_t v;
            } u;
            if constexpr (words >= 4) {
#pragma unroll
                for (int i = 0; i < words; i += 4) {
                    const u32x4 q = __builtin_amdgcn_raw_buffer_load_b128(rows, at + 4 * i, step, 0);
#pragma unroll
                    for (int j = 0; j < 4; ++j) u.w[i + j] = q[j];
                }
            } else {
                const u32x2 q = __builtin_amdgcn_raw_buffer_load_b64(rows, at, step, 0);
                u.w[0] = q[0];
                u.w[1] = q[1];
            }
            v = u.v;
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t at = i < left ? offset + i * (uint32_t)sizeof(T) : kOutside;
                if constexpr (sizeof(T) == 2) v[i] = __builtin_bit_cast(T, (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rows, at, step, 0));
                else v[i] = __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b32(rows, at, step, 0));
            }
        }
    }

    template <bool WIDE> __device__ void store(Rows rows, uint32_t offset, uint32_t step, int left) const
    {
        if constexpr (WIDE) {
            const uint32_t at = left > 0 ? offset : kOutside;
            union {
                uint32_t w[words];
                vec_t v;
            } u;
            u.v = v;
            if constexpr (words >= 4) {
#pragma unroll
                for (int i = 0; i < words; i += 4) {
                    u32x4 q = {u.w[i], u.w[i + 1], u.w[i + 2], u.w[i + 3]};
                    __builtin_amdgcn_raw_buffer_store_b128(q, rows, at + 4 * i, step, 0);
                }
            } else {
                u32x2 q = {u.w[0], u.w[1]};
                __builtin_amdgcn_raw_buffer_store_b64(q, rows, at, step, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t at = i < left ? offset + i * (uint32_t)sizeof(T) : kOutside;
                if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, (T)v[i]), rows, at, step, 0);
                else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, (T)v[i]), rows, at, step, 0);
            }
        }
    }
};

// ---- requests and their states (wpk.h, "sequence layers") ------------------------------------------------
struct Requests {
    const int32_t *starts, *slot_map, *resume;
    int32_t tokens, max_length, slots;
};

// rows [first, first + length) of request i
__device__ inline void request_rows(const Requests &q, int i, int *first, int *length)
{
    if (q.starts) {
        const int a = min(max(q.starts[i], 0), q.tokens), b = min(max(q.starts[i + 1], 0), q.tokens);
        *first = a;
        *length = max(b - a, 0);
    } else {
        *first = i * q.max_length;
        *length = q.max_length;
    }
}

// entry of request i's state, or -1
__device__ inline int request_slot(const Requests &q, int i)
{
    const int s = q.slot_map ? q.slot_map[i] : i;
    return s >= 0 && s < q.slots ? s : -1;
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
