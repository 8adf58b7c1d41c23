// Which kernel computes a product with 4-bit group-scaled weights, for one type of x.
#pragma once

#include "group_gemm.hpp"
#include "group_narrow.hpp"

namespace samd {

template <class X, int NW>
int launch_product(const GroupProduct &p, int words, int groups, hipStream_t s) {
    const int gshift = p.group == 32 ? 5 : p.group == 64 ? 6 : 7;
    if (p.T <= 4 && !p.g8) {
        p.w[0].zero ? launch_vector<X, false, NW>(p, words, groups, gshift, s)
                    : launch_vector<X, true, NW>(p, words, groups, gshift, s);
        return check_launch("group product");
    }
    if (p.T <= 32 && !p.g8)
        return p.w[0].zero ? launch_narrow<X, false, NW>(p, words, groups, s) : launch_narrow<X, true, NW>(p, words, groups, s);
    // More tokens: tiles through LDS.  A workgroup fills a CU, so a tile costs its time for each round of 256
    // workgroups; the units are microseconds measured for K = 4096, groups of 128 (they grow with K alike).
    constexpr int kSlices = sizeof(X) == 4 ? 2 : 4;
    if (!within_buffer(p.x, sizeof(X), std::min<int64_t>(p.T, 256), p.ldx, p.K))
        return launch_gemm_tile<X, false, NW, 2, 4, 2, 1, kSlices>(p, words, groups, s);
    auto cost = [&](int64_t tokens, int64_t rows, int64_t unit) {
        const int64_t blocks = ((p.T + tokens - 1) / tokens) * ((p.M + rows / NW - 1) / (rows / NW));
        return (blocks + 255) / 256 * unit;
    };
    if constexpr (sizeof(X) == 2) {
        const int64_t small = cost(64, 64, 23), middle = cost(128, 128, 53), large = cost(256, 128, 80);
        if (large < middle && large < small) return launch_gemm_tile<X, true, NW, 4, 4, 4, 2, 1>(p, words, groups, s);
        if (middle < small) return launch_gemm_tile<X, true, NW, 4, 4, 2, 2, 2>(p, words, groups, s);
    } else {
        const int64_t small = cost(64, 64, 55), middle = cost(64, 128, 84), large = cost(128, 128, 108);
        if (large < middle && large < small) return launch_gemm_tile<X, true, NW, 2, 4, 4, 2, 1>(p, words, groups, s);
        if (middle < small) return launch_gemm_tile<X, true, NW, 2, 4, 2, 2, 1>(p, words, groups, s);
    }
    return launch_gemm_tile<X, true, NW, 2, 4, 2, 1, kSlices>(p, words, groups, s);
}

template <class X>
int launch_product_of(const GroupProduct &p, hipStream_t s) {
    const int words = (int)row_words(p.K, 4), groups = (p.K + p.group - 1) / p.group;
    return p.act < 0 ? launch_product<X, 1>(p, words, groups, s) : launch_product<X, 2>(p, words, groups, s);
}

}  // namespace samd
