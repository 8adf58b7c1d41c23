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
    if constexpr (sizeof(X) == 2)
        if (p.T > 128) return launch_gemm_tile<X, NW, 4, 4, 4, 2>(p, words, groups, s);
    return launch_gemm_tile<X, NW, 2, 4, 2, 2>(p, words, groups, s);
}

template <class X>
int launch_product_of(const GroupProduct &p, hipStream_t s) {
    const int words = (int)row_words(p.K, 4), groups = (p.K + p.group - 1) / p.group;
    return p.act < 0 ? launch_product<X, 1>(p, words, groups, s) : launch_product<X, 2>(p, words, groups, s);
}

}  // namespace samd
