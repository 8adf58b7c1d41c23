// Device helpers shared by the kernels on group-scaled rows.
#pragma once

#include "hip_util.hpp"

namespace samd {

typedef _Float16 half_t;
typedef __bf16 bf16_t;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Calls f(float{} / half_t{} / bf16_t{}) for an element type; the host has checked the type.
template <class F>
void with_type(int type, F &&f) {
    if (type == SAMD_F32) f(float{});
    else if (type == SAMD_F16) f(half_t{});
    else f(bf16_t{});
}

// Every row of a float matrix starts on 16 bytes.
inline bool rows16(const void *p, int type, int64_t ld) {
    return ((uintptr_t)p & 15) == 0 && (ld * (type == SAMD_F32 ? 4 : 2)) % 16 == 0;
}

// n (at most 8) consecutive values as floats, 0 behind them; `vec`: p is on 16 bytes.
template <class X>
__device__ __forceinline__ void load8(const X *p, int n, bool vec, float (&v)[8]) {
    if (vec && n >= 8) {
        X t[8];
        if constexpr (sizeof(X) == 4) {
            *(u32x4 *)t = *(const u32x4 *)p;
            *(u32x4 *)(t + 4) = *(const u32x4 *)(p + 4);
        } else {
            *(u32x4 *)t = *(const u32x4 *)p;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)t[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? (float)p[i] : 0.0f;
    }
}

template <class X>
__device__ __forceinline__ void store8(X *p, int n, bool vec, const float (&v)[8]) {
    if (vec && n >= 8) {
        X t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = (X)v[i];
        if constexpr (sizeof(X) == 4) {
            *(u32x4 *)p = *(u32x4 *)t;
            *(u32x4 *)(p + 4) = *(u32x4 *)(t + 4);
        } else {
            *(u32x4 *)p = *(u32x4 *)t;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (X)v[i];
    }
}

// A buffer descriptor of `bytes` bytes: reads behind them give 0.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void *p, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, (int)(uint32_t)min(bytes, (int64_t)0xfffffffc), 0x00020000);
}

// Which row an item of a row-major range belongs to: a multiplication where all items are
// below 2^31, a 64-bit division else.
struct RowOf {
    uint32_t per, mul, shift;
    int32_t small;
};

inline RowOf row_of(int64_t items, uint32_t per_row) {
    const Division d = division(per_row);
    return {per_row, d.mul, d.shift, items < ((int64_t)1 << 31)};
}

__device__ __forceinline__ int64_t row_index(const RowOf &r, int64_t item) {
    if (r.small) return (int64_t)(((uint64_t)(uint32_t)item * r.mul) >> r.shift);
    return item / r.per;
}

// A group's step from its span (samd_group_quantize's rule).  `bits` is the largest |x| of the
// group as an integer, which orders infinities and NaN above every number.
struct GroupStep {
    float inv, scale;
    bool bad;
};

__device__ __forceinline__ GroupStep group_step(float span, uint32_t bits, float top, float inv_top) {
    GroupStep s;
    s.bad = bits >= 0x7f800000u || !(span < __builtin_inff());
    const bool none = span < 0x1p-100f;
    s.inv = none || s.bad ? 0.0f : top / span;
    s.scale = s.bad ? __builtin_nanf("") : none ? 0.0f : span * inv_top;
    return s;
}

// The gated block's activation: a = act(g), da = act'(g).  With the 32-bit exponential and
// error function, whose errors of a few units in the last place are far below the type's.
template <int ACT>
__device__ __forceinline__ void activation(float g, float &a, float &da) {
    if constexpr (ACT == SAMD_ACT_SILU) {
        const float p = 1.0f / (1.0f + expf(-g));
        a = g * p;
        da = p * (1.0f + g * (1.0f - p));
    } else {
        const float p = 0.5f * (1.0f + erff(g * 0.70710678118654752f));
        a = g * p;
        da = p + g * expf(-0.5f * g * g) * 0.39894228040143268f;
    }
}

}  // namespace samd
