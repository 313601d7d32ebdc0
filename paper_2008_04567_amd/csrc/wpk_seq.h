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
