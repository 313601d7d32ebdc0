// What the operators around a mixer layer share: rows of eight elements a lane, and 8-bit values with a scale for each 128
// (wpk.h, "around a mixer layer").
#ifndef WPK_Q8_H
#define WPK_Q8_H

#include "wpk_seq.h"

namespace wpk {

// A pass over more bytes than this goes past the caches, which would hold none of it for the next call; of fewer, the next call finds
// its inputs there.  16384 x 4096 bf16 to 8 bits 38 -> 35 us, its norm 95 -> 88; the combination of 4096 x 8 rows of 2048 39 -> 32.  (Each
// measured one call behind the other; what the product that reads such outputs next gains or loses was not.)
static const int64_t kFarBytes = 64 << 20;

static const int kScaleBlock = 128;
static const float kLargest8 = 448.0f, kLeastScale = 0x1p-110f;

inline int64_t scale_blocks(int64_t width) { return (width + kScaleBlock - 1) / kScaleBlock; }

// Eight neighbouring elements, from an address that is aligned to one of them (the device takes such loads and stores).  FAR: past
// the caches.
template <typename T> struct Eight {
    typedef T vec __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    typedef T vec_t __attribute__((ext_vector_type(8)));
    // `left` of them are there; ALL: known to be eight
    template <bool ALL, bool FAR> static __device__ f32x8 load(const T *p, int left)
    {
        if (ALL || left >= 8) {
            if constexpr (FAR) return __builtin_convertvector((vec_t)__builtin_nontemporal_load((const vec *)p), f32x8);
            else return __builtin_convertvector((vec_t) * (const vec *)p, f32x8);
        }
        f32x8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? (float)p[i] : 0.0f;
        return v;
    }
    template <bool ALL, bool FAR> static __device__ void store(T *p, int left, f32x8 v)
    {
        const vec_t u = __builtin_convertvector(v, vec_t);
        if (ALL || left >= 8) {
            if constexpr (FAR) __builtin_nontemporal_store((vec)u, (vec *)p);
            else *(vec *)p = u;
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = u[i];
    }
};

template <int CTRL> __device__ inline float max_with_lane(float v)
{
    const int other = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true);
    return fmaxf(v, __builtin_bit_cast(float, other));
}
// the largest of a row of 16 lanes, in all of them (NaN count as nothing)
__device__ inline float row_max(float v)
{
    v = max_with_lane<0xb1>(v);        // quad_perm 1 0 3 2
    v = max_with_lane<0x4e>(v);        // quad_perm 2 3 0 1
    v = max_with_lane<0x141>(v);       // row_half_mirror
    return max_with_lane<0x140>(v);    // row_mirror
}

// Eight lanes' worth of a block of 128: 16 neighbouring lanes hold it, eight values each, zeros behind its end.  Stores the
// lane's values, and the first lane the scale.  All 16 lanes have to come here.
template <bool ALL, bool FAR> __device__ inline void store_8(uint8_t *q, float *scale, int left, f32x8 v, bool first)
{
    float most = fmaxf(fabsf(v[0]), fabsf(v[1]));
#pragma unroll
    for (int i = 2; i < 8; ++i) most = fmaxf(most, fabsf(v[i]));
    const float s = fmaxf(row_max(most) / kLargest8, kLeastScale), inverse = 1.0f / s;
    v *= inverse;
    u32x2 u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
        u[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], p, true);
    }
    if (ALL || left >= 8) {
        if constexpr (FAR) __builtin_nontemporal_store(u, (u32x2 *)q);
        else *(u32x2 *)q = u;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) q[i] = (uint8_t)(u[i >> 2] >> (8 * (i & 3)));
    }
    if (first && left > 0) *scale = s;
}

}  // namespace wpk
#endif
