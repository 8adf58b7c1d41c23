// Group-scaled rows from float rows and back, and the elementwise half of the gated block's
// backward pass: each value is read once and written once, so all three are bound by HBM.
//
// One thread takes 8 consecutive values: 16 bytes of a 16-bit type, one packed word of 4-bit
// values or two of 8-bit ones.  A group is 4, 8 or 16 neighbouring threads, so its span is two
// to four cross-lane steps and nothing is read twice.
//
// Measured (kernel alone; the call's bytes over its time): 4096 x 4099 f32 to unsigned 4 bits 17.3 us (4.4 TB/s, rows at
// odd addresses), back 15.6 (4.9); 8192 x 4096 bf16 to signed 8 bits 24.6 us (4.2), back 17.9 (5.8, in part from
// cache); the gated gradient of 2048 x 10240 bf16 33.9 us (5.1).  A large copy reaches 5.2.
#include <hip/hip_runtime.h>

#include "group_device.hpp"

namespace samd {

namespace {

constexpr int kBlock = 256;

template <class X, int B, bool SIGNED>
__global__ __launch_bounds__(kBlock) void group_quantize_kernel(const X *__restrict__ src, int64_t items, int32_t cols,
                                                                int64_t ld, int lanes, int words, RowOf div,
                                                                uint32_t *__restrict__ q, float *__restrict__ scale,
                                                                uint8_t *__restrict__ zero) {
    constexpr int kTop = SIGNED ? (1 << (B - 1)) - 1 : (1 << B) - 1;
    const int groups = div.per / lanes;
    // items is a multiple of `lanes` and the stride one of 64: a group's threads run together
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < items; i += (int64_t)gridDim.x * kBlock) {
        const int64_t r = row_index(div, i);
        const uint32_t at = (uint32_t)(i - r * div.per);   // which 8 values of the row, its last group filled up
        const int64_t k0 = (int64_t)at * 8;
        const int n = (int)min((int64_t)8, max((int64_t)0, cols - k0));
        float v[8];
        load8(src + r * ld + k0, n, v);
        uint32_t big = 0;
        float lo = 0.0f, hi = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            big = max(big, __float_as_uint(v[j]) & 0x7fffffffu);
            lo = fminf(lo, v[j]);
            hi = fmaxf(hi, v[j]);
        }
        for (int off = lanes / 2; off > 0; off >>= 1) {
            big = max(big, (uint32_t)__shfl_xor((int)big, off, 64));
            if (!SIGNED) {
                lo = fminf(lo, __shfl_xor(lo, off, 64));
                hi = fmaxf(hi, __shfl_xor(hi, off, 64));
            }
        }
        const GroupStep s = group_step(SIGNED ? __uint_as_float(big) : hi - lo, big, (float)kTop, 1.0f / (float)kTop);
        float z = 0.0f;
        if (!SIGNED && !s.bad) z = fminf(rintf(-lo * s.inv), (float)kTop);
        uint32_t f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float t = fminf(fmaxf(rintf(v[j] * s.inv) + z, SIGNED ? -(float)kTop : 0.0f), (float)kTop);
            // fields behind the row's end stay 0 (an unsigned 0 is stored as its zero point)
            f[j] = s.bad || j >= n ? 0u : (uint32_t)(int)t & ((1u << B) - 1);
        }
        if (n > 0) {
            if constexpr (B == 4) {
                uint32_t w = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) w |= f[j] << (4 * j);
                q[r * words + at] = w;
            } else {
                const uint32_t w0 = f[0] | f[1] << 8 | f[2] << 16 | f[3] << 24;
                const uint32_t w1 = f[4] | f[5] << 8 | f[6] << 16 | f[7] << 24;
                uint32_t *d = q + r * words + 2 * (int64_t)at;
                if (words % 2 == 0 && ((uintptr_t)q & 7) == 0) {
                    *(u32x2 *)d = u32x2{w0, w1};
                } else {
                    d[0] = w0;
                    if (n > 4) d[1] = w1;
                }
            }
        }
        if (at % lanes == 0) {
            const int64_t g = r * groups + at / lanes;
            scale[g] = s.scale;
            if (!SIGNED) zero[g] = (uint8_t)z;
        }
    }
}

// The 8 whole values of item `at` of a packed row (n of them in the row).
template <int B>
__device__ __forceinline__ void load_fields(const uint32_t *row, int64_t at, int n, bool vec, uint32_t (&f)[8]) {
    if constexpr (B == 4) {
        const uint32_t w = row[at];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = (w >> (4 * j)) & 15u;
    } else {
        u32x2 w;
        if (vec) {
            w = *(const u32x2 *)(row + 2 * at);
        } else {
            w[0] = row[2 * at];
            w[1] = n > 4 ? row[2 * at + 1] : 0u;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = (w[j / 4] >> (8 * (j % 4))) & 255u;
    }
}

template <int B, bool SIGNED>
__device__ __forceinline__ float field_value(uint32_t f, int z) {
    if (SIGNED) return (float)((int)(f << (32 - B)) >> (32 - B));
    return (float)((int)f - z);
}

template <class X, int B, bool SIGNED>
__global__ __launch_bounds__(kBlock) void group_dequantize_kernel(const uint32_t *__restrict__ q,
                                                                  const float *__restrict__ scale,
                                                                  const uint8_t *__restrict__ zero, int64_t items,
                                                                  int32_t cols, int words, int groups, int gshift,
                                                                  RowOf div, X *__restrict__ dst, int64_t ld,
                                                                  bool vecq) {
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < items; i += (int64_t)gridDim.x * kBlock) {
        const int64_t r = row_index(div, i);
        const int64_t at = i - r * div.per, k0 = at * 8;
        const int n = (int)min((int64_t)8, cols - k0);
        const int64_t g = r * groups + (k0 >> gshift);
        const float s = scale[g];
        const int z = SIGNED ? 0 : (int)zero[g];
        uint32_t f[8];
        load_fields<B>(q + r * words, at, n, vecq, f);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = s * field_value<B, SIGNED>(f[j], z);
        store8(dst + r * ld + k0, n, v);
    }
}

template <class X>
__global__ __launch_bounds__(kBlock) void group_gated_grad_kernel(const X *__restrict__ dh, int64_t lddh, GroupW g,
                                                                  GroupW u, int64_t items, int32_t M, int words,
                                                                  int groups, int gshift, RowOf div,
                                                                  X *__restrict__ dg, X *__restrict__ du, int64_t ldd,
                                                                  int act, bool vecq) {
    for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < items; i += (int64_t)gridDim.x * kBlock) {
        const int64_t r = row_index(div, i);
        const int64_t at = i - r * div.per, k0 = at * 8;
        const int n = (int)min((int64_t)8, M - k0);
        const int64_t s = r * groups + (k0 >> gshift);
        uint32_t fg[8], fu[8];
        load_fields<8>(g.q + r * words, at, n, vecq, fg);
        load_fields<8>(u.q + r * words, at, n, vecq, fu);
        const float sg = g.scale[s], su = u.scale[s];
        float d[8], a[8], b[8];
        load8(dh + r * lddh + k0, n, d);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float value, slope;
            activation(act, sg * field_value<8, true>(fg[j], 0), value, slope);
            a[j] = d[j] * (su * field_value<8, true>(fu[j], 0)) * slope;
            b[j] = d[j] * value;
        }
        store8(dg + r * ldd + k0, n, a);
        store8(du + r * ldd + k0, n, b);
    }
}

inline int group_shift(int group) { return group == 32 ? 5 : group == 64 ? 6 : 7; }

}  // namespace

int launch_group_quantize(const void *src, int type, int64_t rows, int64_t cols, int64_t ld, samd_fmt f, int group,
                          uint32_t *q, float *scale, uint8_t *zero, hipStream_t s) {
    const int64_t groups = (cols + group - 1) / group;
    const int lanes = group / 8;
    const int64_t items = rows * groups * lanes;
    const int grid = grid_for(items, kBlock);
    const int words = (int)row_words(cols, f.bits);
    const RowOf div = row_of(items, (uint32_t)(groups * lanes));
    with_type(type, [&](auto t) {
        using X = decltype(t);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(grid), dim3(kBlock), 0, s, (const X *)src, items, (int32_t)cols, ld, lanes,
                               words, div, q, scale, zero);
        };
        if (f.bits == 4) f.is_signed ? go(group_quantize_kernel<X, 4, true>) : go(group_quantize_kernel<X, 4, false>);
        else f.is_signed ? go(group_quantize_kernel<X, 8, true>) : go(group_quantize_kernel<X, 8, false>);
    });
    return check_launch("samd_group_quantize");
}

int launch_group_dequantize(const GroupW &w, int64_t rows, int64_t cols, samd_fmt f, int group, void *dst, int type,
                            int64_t ld, hipStream_t s) {
    const int64_t groups = (cols + group - 1) / group, per = (cols + 7) / 8;
    const int64_t items = rows * per;
    const int grid = grid_for(items, kBlock);
    const int words = (int)row_words(cols, f.bits);
    const RowOf div = row_of(items, (uint32_t)per);
    const bool vecq = words % 2 == 0 && ((uintptr_t)w.q & 7) == 0;
    with_type(type, [&](auto t) {
        using X = decltype(t);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(grid), dim3(kBlock), 0, s, w.q, w.scale, w.zero, items, (int32_t)cols,
                               words, (int)groups, group_shift(group), div, (X *)dst, ld, vecq);
        };
        if (f.bits == 4)
            f.is_signed ? go(group_dequantize_kernel<X, 4, true>) : go(group_dequantize_kernel<X, 4, false>);
        else
            f.is_signed ? go(group_dequantize_kernel<X, 8, true>) : go(group_dequantize_kernel<X, 8, false>);
    });
    return check_launch("samd_group_dequantize");
}

int launch_group_gated_grad(const void *dh, int type, int64_t lddh, const GroupW &g, const GroupW &u, int group, int act,
                            int64_t T, int64_t M, void *dg, void *du, int64_t ldd, hipStream_t s) {
    const int64_t groups = (M + group - 1) / group, per = (M + 7) / 8;
    const int64_t items = T * per;
    const int grid = grid_for(items, kBlock);
    const int words = (int)row_words(M, 8);
    const RowOf div = row_of(items, (uint32_t)per);
    const bool vecq = words % 2 == 0 && (((uintptr_t)g.q | (uintptr_t)u.q) & 7) == 0;
    with_type(type, [&](auto t) {
        using X = decltype(t);
        hipLaunchKernelGGL((group_gated_grad_kernel<X>), dim3(grid), dim3(kBlock), 0, s, (const X *)dh, lddh, g, u, items,
                           (int32_t)M, words, (int)groups, group_shift(group), div, (X *)dg, (X *)du, ldd, act, vecq);
    });
    return check_launch("samd_group_gated_grad");
}

}  // namespace samd
