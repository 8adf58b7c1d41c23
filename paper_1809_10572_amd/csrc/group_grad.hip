// The input gradient of products with 4-bit group-scaled weights: dx = dy W (+ dy2 W2).
//
// One thread computes 8 consecutive columns of one token, walking the rows of W.
#include <hip/hip_runtime.h>

#include "group_device.hpp"

namespace samd {

namespace {

template <class X>
__global__ __launch_bounds__(256) void group_grad_kernel(GroupGrad p, int words, int groups, int gshift, int64_t items,
                                                         RowOf div) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= items) return;
    const int64_t t = row_index(div, i);
    const int w = (int)(i - t * div.per);
    float acc[8] = {};
    for (int a = 0; a < 2 && p.dy[a]; ++a) {
        const X *dy = (const X *)p.dy[a] + t * p.lddy;
        for (int m = 0; m < p.M; ++m) {
            const int64_t g = (int64_t)m * groups + (w >> (gshift - 3));
            const uint32_t q = p.w[a].q[(int64_t)m * words + w];
            const int z = p.w[a].zero ? (int)p.w[a].zero[g] : 8;
            const uint32_t u = p.w[a].zero ? q : q ^ 0x88888888u;
            const float v = (float)dy[m];
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += v * (p.w[a].scale[g] * (float)((int)((u >> (4 * j)) & 15u) - z));
        }
    }
    store8((X *)p.dx + t * p.lddx + (int64_t)w * 8, min(8, p.K - w * 8), false, acc);
}

}  // namespace

int launch_group_matmul_grad(const GroupGrad &p, hipStream_t s) {
    const int words = (int)row_words(p.K, 4), groups = (p.K + p.group - 1) / p.group;
    const int gshift = p.group == 32 ? 5 : p.group == 64 ? 6 : 7;
    const int64_t items = (int64_t)p.T * words;
    if ((items + 255) / 256 > INT32_MAX) {
        set_error("samd_group_matmul_grad: T x K needs too many workgroups");
        return SAMD_EUNSUPPORTED;
    }
    const RowOf div = row_of(items, (uint32_t)words);
    with_type(p.type, [&](auto t) {
        using X = decltype(t);
        hipLaunchKernelGGL((group_grad_kernel<X>), dim3((uint32_t)((items + 255) / 256)), dim3(256), 0, s, p, words, groups,
                           gshift, items, div);
    });
    return check_launch("samd_group_matmul_grad");
}

}  // namespace samd
