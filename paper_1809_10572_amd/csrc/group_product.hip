// Products of float activations with 4-bit group-scaled weights, y = x W^T, and the gated block on
// two of them: h = act(x Wg^T) * (x Wu^T).
//
// One workgroup computes 32 consecutive rows of W (one stored group of the gated block) for 4
// tokens: every wave 8 rows, its lanes along K.  A weight's whole value is multiplied exactly;
// a word's sum of 8 products is scaled once, in 32-bit floats.
#include <hip/hip_runtime.h>

#include "group_vector.hpp"

namespace samd {

namespace {

constexpr int kTokens = 4, kRows = 32;

template <class X, int ACT>   // ACT -1: the product alone
__global__ __launch_bounds__(256) void group_product_kernel(GroupProduct p, int words, int groups, int gshift) {
    constexpr int NW = ACT < 0 ? 1 : 2;
    __shared__ float sum[NW][kTokens][kRows];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int mblocks = (p.M + kRows - 1) / kRows;
    const int m0 = (int)(blockIdx.x % mblocks) * kRows, t0 = (int)(blockIdx.x / mblocks) * kTokens;
    for (int j = wave * 8; j < wave * 8 + 8; ++j) {
        const int m = min(m0 + j, p.M - 1);
        float acc[NW][kTokens] = {};
        for (int w = lane; w < words; w += 64) {
            float x[kTokens][8];
#pragma unroll
            for (int t = 0; t < kTokens; ++t) {
                const X *row = (const X *)p.x + (int64_t)min(t0 + t, p.T - 1) * p.ldx;
                load8(row + (int64_t)w * 8, min(8, p.K - w * 8), false, x[t]);
            }
#pragma unroll
            for (int a = 0; a < NW; ++a) {
                const int64_t g = (int64_t)m * groups + (w >> (gshift - 3));
                const uint32_t q = p.w[a].q[(int64_t)m * words + w];
                const float s = p.w[a].scale[g];
                const int z = p.w[a].zero ? (int)p.w[a].zero[g] : 8;
                const uint32_t u = p.w[a].zero ? q : q ^ 0x88888888u;
                float part[kTokens] = {};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float v = (float)((int)((u >> (4 * i)) & 15u) - z);
#pragma unroll
                    for (int t = 0; t < kTokens; ++t) part[t] += v * x[t][i];
                }
#pragma unroll
                for (int t = 0; t < kTokens; ++t) acc[a][t] += s * part[t];
            }
        }
#pragma unroll
        for (int a = 0; a < NW; ++a)
#pragma unroll
            for (int t = 0; t < kTokens; ++t) {
                float v = acc[a][t];
                for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
                if (lane == 0) sum[a][t][j] = v;
            }
    }
    __syncthreads();
    if (threadIdx.x >= kTokens * kRows) return;
    const int t = threadIdx.x / kRows, j = threadIdx.x % kRows;
    const bool in = t0 + t < p.T && m0 + j < p.M;
    float out = sum[0][t][j];
    if constexpr (ACT >= 0) {
        const float g = sum[0][t][j], u = sum[1][t][j];
        float da;
        activation<ACT>(g, out, da);
        out *= u;
        if (p.g8) {   // the 32 threads of a token are one stored group
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                const float v = in ? (a ? u : g) : 0.0f;
                uint32_t big = __float_as_uint(v) & 0x7fffffffu;
                for (int off = 16; off > 0; off >>= 1) big = max(big, (uint32_t)__shfl_xor((int)big, off, 64));
                const GroupStep s = group_step(__uint_as_float(big), big, 127.0f, 1.0f / 127.0f);
                uint32_t f = s.bad ? 0u : (uint32_t)(int)rintf(v * s.inv) & 255u;
                f <<= 8 * (j & 3);
                f |= (uint32_t)__shfl_xor((int)f, 1, 64);
                f |= (uint32_t)__shfl_xor((int)f, 2, 64);
                const int saved_words = (p.M + 3) / 4, saved_groups = mblocks;
                if (in && j % 4 == 0) (a ? p.u8 : p.g8)[(int64_t)(t0 + t) * saved_words + (m0 + j) / 4] = f;
                if (in && j == 0) (a ? p.uscale : p.gscale)[(int64_t)(t0 + t) * saved_groups + m0 / kRows] = s.scale;
            }
        }
    }
    if (in) ((X *)p.y)[(int64_t)(t0 + t) * p.ldy + m0 + j] = (X)out;
}

}  // namespace

int launch_group_product(const GroupProduct &p, hipStream_t s) {
    const int words = (int)row_words(p.K, 4), groups = (p.K + p.group - 1) / p.group;
    const int gshift = p.group == 32 ? 5 : p.group == 64 ? 6 : 7;
    if (p.T <= 4 && !p.g8) {
        with_type(p.type, [&](auto t) {
            using X = decltype(t);
            auto go = [&](auto is_signed) {
                constexpr bool S = decltype(is_signed)::value;
                if (p.act < 0) launch_vector<X, S, 1, -1>(p, words, groups, gshift, s);
                else if (p.act == SAMD_ACT_SILU) launch_vector<X, S, 2, SAMD_ACT_SILU>(p, words, groups, gshift, s);
                else launch_vector<X, S, 2, SAMD_ACT_GELU>(p, words, groups, gshift, s);
            };
            p.w[0].zero ? go(std::false_type{}) : go(std::true_type{});
        });
        return check_launch("group product");
    }
    const int64_t blocks = (((int64_t)p.M + kRows - 1) / kRows) * (((int64_t)p.T + kTokens - 1) / kTokens);
    if (blocks > INT32_MAX) {
        set_error("group product: T x M needs too many workgroups");
        return SAMD_EUNSUPPORTED;
    }
    with_type(p.type, [&](auto t) {
        using X = decltype(t);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(256), 0, s, p, words, groups, gshift);
        };
        if (p.act < 0) go(group_product_kernel<X, -1>);
        else if (p.act == SAMD_ACT_SILU) go(group_product_kernel<X, SAMD_ACT_SILU>);
        else go(group_product_kernel<X, SAMD_ACT_GELU>);
    });
    return check_launch("group product");
}

}  // namespace samd
