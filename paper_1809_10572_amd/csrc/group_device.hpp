// Device helpers shared by the kernels on group-scaled rows.
#pragma once

#include "hip_util.hpp"

namespace samd {

typedef _Float16 half_t;
typedef __bf16 bf16_t;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef half_t half2_t __attribute__((ext_vector_type(2)));
typedef bf16_t bf162_t __attribute__((ext_vector_type(2)));

// Calls f(float{} / half_t{} / bf16_t{}) for an element type; the host has checked the type.
template <class F>
void with_type(int type, F &&f) {
    if (type == SAMD_F32) f(float{});
    else if (type == SAMD_F16) f(half_t{});
    else f(bf16_t{});
}

// v, of which the compiler knows nothing: bytes of a masked word are converted to floats where they stand,
// not cut out first.
__device__ __forceinline__ uint32_t as_is(uint32_t v) {
    asm("" : "+v"(v));
    return v;
}

// v as a 32-bit float: a product that is stored as f16 would be rounded to it at once, not to float first as defined.
__device__ __forceinline__ float as_float(float v) {
    asm("" : "+v"(v));
    return v;
}

// 16 and 8 bytes at the alignment of an element of 2 or 4: global memory takes them in one access all the same.  (As
// words, not as elements: the compiler would take stores of the last element out of both branches below.)
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));
typedef u32x2 u32x2_at2 __attribute__((aligned(2)));
template <class X>
using Bytes16 = std::conditional_t<sizeof(X) == 4, u32x4_at4, u32x4_at2>;

// 8 values, and the same as words.
template <class X>
struct Eight {
    X v[8];
};
template <class X>
struct Raw8 {
    u32x4 v[sizeof(X) / 2];
};

// 8 consecutive values as they are stored, n of them in the row (at most; 0 behind them).
template <class X>
__device__ __forceinline__ Raw8<X> raw8(const X *p, int n) {
    Raw8<X> r;
    if (n >= 8) {
#pragma unroll
        for (int h = 0; h < (int)sizeof(X) / 2; ++h) r.v[h] = ((const Bytes16<X> *)p)[h];
    } else {
        Eight<X> t;
#pragma unroll
        for (int i = 0; i < 8; ++i) t.v[i] = i < n ? p[i] : (X)0.0f;
        r = __builtin_bit_cast(Raw8<X>, t);
    }
    return r;
}

// The same as floats.
template <class X>
__device__ __forceinline__ void load8(const X *p, int n, float (&v)[8]) {
    const Eight<X> t = __builtin_bit_cast(Eight<X>, raw8(p, n));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)t.v[i];
}

template <class X>
__device__ __forceinline__ void store8(X *p, int n, const float (&v)[8]) {
    Eight<X> t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t.v[i] = (X)as_float(v[i]);
    if (n >= 8) {
        const Raw8<X> w = __builtin_bit_cast(Raw8<X>, t);
#pragma unroll
        for (int h = 0; h < (int)sizeof(X) / 2; ++h) ((Bytes16<X> *)p)[h] = w.v[h];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = t.v[i];
    }
}

// A buffer descriptor of `bytes` bytes from p on, which is on 4 bytes, filled up to a whole word (a word that holds the
// last value is read whole, from within one page): reads of words behind them give 0.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void *p, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, (int)(uint32_t)min((bytes + 3) & ~(int64_t)3, (int64_t)0xfffffffc),
                                             0x00020000);
}

// The same for zero points, which are read by bytes and may start anywhere: exactly those bytes, since the words that
// they are filled up to from such a start could reach into another page.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t byte_buffer_of(const uint8_t *p, int64_t bytes) {
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

// The 8 fields of a word less their zero point as 16-bit floats, exactly: pairs of fields i and i + 4, i = 0 .. 3.  A field
// put under the bits of 1024 is 1024 + u (one that stands four bits higher, 1024 + 16 u); the rest is a subtraction of
// whole numbers, or a multiply-add with 1/16.  Signed fields have their sign bit flipped: u is the value plus 8.
struct ZeroPoint {
    half2_t less, less16;   // -(1024 + z), -(64 + z)
};
template <bool SIGNED>
__device__ __forceinline__ ZeroPoint zero_point(uint32_t z) {   // of 0 .. 255
    if (SIGNED) z = 8;
    const half2_t at1024 = __builtin_bit_cast(half2_t, z * 0x00010001u + 0x64006400u);
    const half2_t k960 = {(half_t)960.0f, (half_t)960.0f};
    return {-at1024, k960 - at1024};
}

// -(1024 + z) and -(64 + z) in one word.
template <bool SIGNED>
__device__ __forceinline__ float zero_point_word(uint32_t z) {
    const ZeroPoint p = zero_point<SIGNED>(z);
    return __uint_as_float(__builtin_bit_cast(uint32_t, half2_t{p.less[0], p.less16[0]}));
}

// The fields as such, put under bits: 1024 + u in [0] and [2], 1024 + 16 u in [1] and [3].
template <bool SIGNED>
__device__ __forceinline__ void field_pairs(uint32_t w, half2_t (&out)[4]) {
    // as unknown values, so that `and` and `xor` with them are one operation
    const uint32_t one = as_is(SIGNED ? 0x64086408u : 0x64006400u), sixteen = SIGNED ? as_is(0x64806480u) : one;
    const uint32_t v = w >> 8;
    out[0] = __builtin_bit_cast(half2_t, (w & 0x000f000fu) ^ one);
    out[1] = __builtin_bit_cast(half2_t, (w & 0x00f000f0u) ^ sixteen);
    out[2] = __builtin_bit_cast(half2_t, (v & 0x000f000fu) ^ one);
    out[3] = __builtin_bit_cast(half2_t, (v & 0x00f000f0u) ^ sixteen);
}

template <bool SIGNED>
__device__ __forceinline__ void whole_pairs(uint32_t w, const ZeroPoint &z, half2_t (&out)[4]) {
    const half2_t sixteenth = {(half_t)0.0625f, (half_t)0.0625f};
    field_pairs<SIGNED>(w, out);
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        out[i] += z.less;
        out[i + 1] = __builtin_elementwise_fma(out[i + 1], sixteenth, z.less16);
    }
}

// The same as a matrix operand of f16 or bf16, whose 8 bits hold every difference of 4 bits and a byte too: each difference
// by one multiply-add from f16 to f32, the upper halves of two.
template <class H, bool SIGNED>
__device__ __forceinline__ u32x4 whole_operand(uint32_t w, const ZeroPoint &z) {
    half2_t v[4];
    u32x4 out;
    if constexpr (std::is_same_v<H, half_t>) {
        whole_pairs<SIGNED>(w, z, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i] = __builtin_bit_cast(uint32_t, v[i]);
    } else {
        field_pairs<SIGNED>(w, v);
        const float one = as_float(1.0f);   // an unknown value: the multiply-add reads f16, an addition would not
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const half2_t less = i % 2 ? z.less16 : z.less;
            const float k = i % 2 ? 0.0625f : one;
            const float lo = fmaf((float)v[i][0], k, (float)less[0]), hi = fmaf((float)v[i][1], k, (float)less[1]);
            out[i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
        }
    }
    return out;
}

// The gated block's activation: a = act(g), da = act'(g), with the 32-bit exponential and complementary error function;
// values next to 0 keep their relative accuracy.  erfc(-g / sqrt 2), not 1 + erf: that cancels for negative g (off by 4 %
// at -5, 0 from -5.5 on).  What the argument's rounding leaves grows with g^2: 1.5 (g^2 + 1) + 36 units of 2^-24 of the
// value, 16 last places of the function in them.
__device__ __forceinline__ void activation(int act, float g, float &a, float &da) {
    if (act == SAMD_ACT_SILU) {
        const float e = expf(-fabsf(g)), p = (g < 0.0f ? e : 1.0f) / (1.0f + e);   // e^-g overflows from -88.7 on
        a = g * p;
        da = p * (1.0f + g * (1.0f - p));
    } else {
        const float p = 0.5f * erfcf(g * -0.70710678118654752f);
        a = g * p;
        da = p + g * expf(-0.5f * g * g) * 0.39894228040143268f;
    }
}

typedef half_t half8_t __attribute__((ext_vector_type(8)));
typedef bf16_t bf168_t __attribute__((ext_vector_type(8)));

// D = A B + C on 16 x 16 x 32; operands as four words of two 16-bit floats.
template <class X>
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (std::is_same_v<X, half_t>)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf168_t, a), __builtin_bit_cast(bf168_t, b), c, 0, 0, 0);
}

// 16-bit pieces of 8 activations: the values themselves, or three bf16 pieces of 32-bit ones.
template <class X>
constexpr int kPieces = sizeof(X) == 4 ? 3 : 1;

// Zeroes behind the first n.
template <class X>
__device__ __forceinline__ void clear_behind(Raw8<X> &r, int n) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if constexpr (sizeof(X) == 4) r.v[j / 4][j % 4] = j < n ? r.v[j / 4][j % 4] : 0u;
        else r.v[0][j / 2] &= j < n ? 0xffffffffu : j % 2 ? 0x0000ffffu : 0u;
    }
}

// The matrix operands of 8 values, in their order.  A 32-bit value goes into three bf16 pieces: its upper 8
// significant bits, the next 8, the last 8, each by cutting the rest off, so that they add up to it.
template <class X>
__device__ __forceinline__ void x_operand(const Raw8<X> &raw, u32x4 (&out)[kPieces<X>]) {
    if constexpr (sizeof(X) == 4) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(raw.v[i / 4][i % 4]);
#pragma unroll
        for (int j = 0; j < 3; ++j) {
#pragma unroll
            for (int i = 0; i < 4; ++i)   // the upper halves of two values
                out[j][i] = __builtin_amdgcn_perm(__float_as_uint(v[2 * i + 1]), __float_as_uint(v[2 * i]), 0x07060302u);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] -= __uint_as_float(__float_as_uint(v[i]) & 0xffff0000u);
        }
    } else {
        out[0] = raw.v[0];
    }
}

// The same in the order in which pairs of fields come out of a word: 0, 4, 1, 5, 2, 6, 3, 7.
template <class X>
__device__ __forceinline__ void x_operand_paired(const Raw8<X> &raw, u32x4 (&out)[kPieces<X>]) {
    x_operand(raw, out);
#pragma unroll
    for (int j = 0; j < kPieces<X>; ++j) {
        const u32x4 w = out[j];
        out[j] = u32x4{__builtin_amdgcn_perm(w[2], w[0], 0x05040100u), __builtin_amdgcn_perm(w[2], w[0], 0x07060302u),
                       __builtin_amdgcn_perm(w[3], w[1], 0x05040100u), __builtin_amdgcn_perm(w[3], w[1], 0x07060302u)};
    }
}

// Whether a launch of `blocks` workgroups is possible: below 2^32 threads.
inline int check_blocks(int64_t blocks, int threads, const char *call) {
    if (blocks > UINT32_MAX / threads) {
        set_error(std::string(call) + ": a result of so many values needs 2^32 threads or more in one launch");
        return SAMD_EUNSUPPORTED;
    }
    return SAMD_OK;
}

// Whether `rows` rows can be read through one buffer descriptor: on 4 bytes and within 4 GB.
inline bool within_buffer(const void *p, int64_t size, int64_t rows, int64_t ld, int64_t cols) {
    return ((uintptr_t)p & 3) == 0 && ld * size % 4 == 0 && ((__int128)rows * ld + cols) * size < (__int128)0xff000000;
}

}  // namespace samd
