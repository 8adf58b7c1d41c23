// Which kernel computes a product with 4-bit group-scaled weights, for one type of x.
#pragma once

#include "group_gemm.hpp"
#include "group_narrow.hpp"

namespace samd {

// NW 1: the product; 2: the gated block on two.
template <class X, int NW>
int launch_product(const GroupProduct &p, hipStream_t s) {
    const int words = (int)row_words(p.K, 4), groups = (p.K + p.group - 1) / p.group;
    const int gshift = p.group == 32 ? 5 : p.group == 64 ? 6 : 7;
    // One or two tokens: a row of W a wave (two tokens 4096 x 4096: 5.9 us, on the matrix cores 6.0; 8192 x 8192 unsigned
    // groups of 64 15.5 and 17.3; 16384 x 8192, even: 24.2 and 23.7).  The lanes' operations grow with the tokens, the matrix
    // cores take three and four in the time of one.
    if (p.T <= 2 && !p.g8) {
        return p.w[0].zero ? launch_vector<X, false, NW>(p, words, groups, gshift, s)
                           : launch_vector<X, true, NW>(p, words, groups, gshift, s);
    }
    // Up to 16: one operand of tokens, W from memory into operands.
    if (p.T <= 16 && !p.g8)
        return p.w[0].zero ? launch_narrow<X, false, NW>(p, words, groups, s) : launch_narrow<X, true, NW>(p, words, groups, s);
    // More tokens.  A workgroup fills a CU, so a kernel costs its time for each round of 256 workgroups; the units are
    // about the microseconds measured for K = 4096, groups of 128 (they grow with K alike; groups of 32 take up to a quarter
    // more, each kernel).  Rows of x at odd addresses, an odd K of a 16-bit type, have the smallest tile alone: 2048 x 4096 x
    // 4095 bf16 takes 246 us where 4096 takes 84.
    auto cost = [&](int64_t tokens, int64_t rows, int64_t unit) {
        const int64_t blocks = ((p.T + tokens - 1) / tokens) * ((p.M + rows - 1) / rows);
        return (blocks + 255) / 256 * unit;
    };
    constexpr bool kWide = sizeof(X) == 4;
    constexpr int kSlices = kWide ? 2 : 4;
    const bool buffered = within_buffer(p.x, sizeof(X), std::min<int64_t>(p.T, 256), p.ldx, p.K);
    int64_t narrow = p.g8 ? INT64_MAX / 2 : cost(32, 16, (kWide ? 23 : 11) + (NW > 1 ? (kWide ? 12 : 6) : 0));
    if (!buffered) narrow *= 2;   // rows of x at odd addresses: 100 x 2001 x 1501 takes it 21 us, a tile 17
    const int64_t small = cost(64, 64 / NW, kWide ? 55 : 23);
    const int64_t middle = kWide ? cost(64, 128 / NW, 84) : cost(128, 128 / NW, 53);
    const int64_t large = kWide ? cost(128, 128 / NW, 108) : cost(256, 128 / NW, 85);
    if (narrow < std::min(small, std::min(middle, large)))
        return p.w[0].zero ? launch_narrow<X, false, NW>(p, words, groups, s) : launch_narrow<X, true, NW>(p, words, groups, s);
    if (!buffered)
        return launch_gemm_tile<X, false, NW, 2, 4, 2, 1, kSlices>(p, words, groups, s);
    if constexpr (!kWide) {
        if (large < std::min(small, middle)) return launch_gemm_tile<X, true, NW, 4, 4, 4, 2, 1>(p, words, groups, s);
        if (middle < small) return launch_gemm_tile<X, true, NW, 4, 4, 2, 2, 2>(p, words, groups, s);
    } else {
        if (large < std::min(small, middle)) return launch_gemm_tile<X, true, NW, 2, 4, 4, 2, 1>(p, words, groups, s);
        if (middle < small) return launch_gemm_tile<X, true, NW, 2, 4, 2, 2, 1>(p, words, groups, s);
    }
    return launch_gemm_tile<X, true, NW, 2, 4, 2, 1, kSlices>(p, words, groups, s);
}

}  // namespace samd
