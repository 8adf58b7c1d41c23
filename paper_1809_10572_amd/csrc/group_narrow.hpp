// Products of some tens of tokens with 4-bit group-scaled weights on the matrix cores.
//
// The weights still come from memory once, so they go straight into the registers that the
// 16 x 16 x 32 matrix instruction reads: lane l holds row l % 16 of W, quarter l / 16 of the values that one
// instruction sums over.  A step is 128 values of a row, 16 words, four neighbouring ones to a lane; which of them an
// instruction takes is free as long as both operands agree and all lie in one group, so groups of 128 need no
// exchange, groups of 64 and 32 one or two exchanges between halves and rows of lanes (PER = group / 32 instructions
// a group).  A field becomes the 16-bit float u - z exactly, by one to two operations; a group's sum is scaled once, in
// 32-bit floats.
// 32-bit activations enter as three bf16 pieces of 8 bits each, which hold all 24 bits: the products stay
// exact, three instructions for each.
//
// A workgroup computes 16 MT rows of W for 16 TT tokens, its eight waves taking steps of K in turn; their
// sums meet in LDS in a fixed order.
//
// Bound by the latency of a wave's few steps and by what each CU reads through L1: 16 x 4096 x 4096 bf16 takes 8.5 us
// (signed groups of 128), 16 x 8192 x 8192 22 us, against 1.8 and 7 for reading the weights once at 5.2 TB/s.  (f16, unsigned
// groups of 64, 4096 x 4096, counted: half of the waves' cycles are waits, 15400 accesses of a CU's L1 in some 21000 cycles.)
#pragma once

#include "group_vector.hpp"

namespace samd {

constexpr int kNarrowWaves = 8;

// The upper 32 lanes of w[A] and the lower 32 of w[B] change places; within each half, the upper 16 lanes of w[A] and the
// lower 16 of w[B].
template <int A, int B>
__device__ __forceinline__ void swap_halves(u32x4 &w) {
    const auto r = __builtin_amdgcn_permlane32_swap(w[A], w[B], false, false);
    w[A] = r[0], w[B] = r[1];
}
template <int A, int B>
__device__ __forceinline__ void swap_rows(u32x4 &w) {
    const auto r = __builtin_amdgcn_permlane16_swap(w[A], w[B], false, false);
    w[A] = r[0], w[B] = r[1];
}

template <class X, bool SIGNED, int PER, int TT, int NW, int MT>
__global__ __launch_bounds__(64 * kNarrowWaves) void group_narrow_kernel(GroupProduct p, int words, int groups,
                                                                         bool buffered, bool whole_zeros) {
    constexpr int kGroups = 4 / PER;   // groups of a step
    constexpr int kTokens = 16 * TT, kRows = 16 * MT;
    constexpr int NR = NW * MT;   // 16-row sets: set r is rows r % MT * 16 .. of matrix r / MT
    using H = std::conditional_t<std::is_same_v<X, half_t>, half_t, bf16_t>;
    constexpr int kPart = NR * TT * 4;   // sums of a lane
    __shared__ float meet[kNarrowWaves * kPart * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int quarter = lane >> 4, low = lane & 15;
    const int mblocks = (int)(((int64_t)p.M + kRows - 1) / kRows);
    const int64_t m0 = (int64_t)(blockIdx.x % mblocks) * kRows, t0 = (int64_t)(blockIdx.x / mblocks) * kTokens;
    const int rows = (int)min((int64_t)kRows, p.M - m0), tokens = (int)min((int64_t)kTokens, p.T - t0);
    const int steps = (p.K + 127) / 128;

    // Reads behind W's end give 0; what a row's last step reads of the next row meets an x of 0.
    __amdgpu_buffer_rsrc_t rq[NW], rs[NW], rz[NW];
#pragma unroll
    for (int a = 0; a < NW; ++a) {
        rq[a] = buffer_of(p.w[a].q + m0 * words, (int64_t)rows * words * 4);
        rs[a] = buffer_of(p.w[a].scale + m0 * groups, (int64_t)rows * groups * 4);
        rz[a] = byte_buffer_of(p.w[a].zero + m0 * groups, SIGNED ? 0 : (int64_t)rows * groups);
    }
    uint32_t qrow[MT], srow[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const uint32_t r = (uint32_t)min(m * 16 + low, rows - 1);
        qrow[m] = r * (uint32_t)words, srow[m] = r * (uint32_t)groups;
    }
    struct Step {
        u32x4 w[NR];
        float s[NR][kGroups];
        uint32_t z[NR];   // a byte for each group
        Raw8<X> x[TT][4];
    };
    // the 8 values of a row of x that instruction i of a step takes in this lane (i / PER is the group)
    auto k_of = [&](int step, int i) {
        const int word = PER == 4 ? quarter * 4 + i : PER == 2 ? i / 2 * 8 + quarter % 2 * 4 + quarter / 2 * 2 + i % 2 : i * 4 + quarter;
        return step * 128 + word * 8;
    };
    // A lane's four neighbouring words to those of instructions 0 .. 3.
    auto by_instruction = [](u32x4 &w) {
        if constexpr (PER <= 2) {
            swap_halves<0, 2>(w);
            swap_halves<1, 3>(w);
        }
        if constexpr (PER == 1) {
            swap_rows<0, 1>(w);
            swap_rows<2, 3>(w);
        }
    };

    f32x4 acc[NR][TT] = {};
    // BUF: rows of x on 4 bytes, within 4 GB of each other: read through one descriptor, any 4-byte alignment
    auto body = [&](auto buf) {
        constexpr bool BUF = decltype(buf)::value;
        const __amdgpu_buffer_rsrc_t rx = buffer_of((const X *)p.x + t0 * p.ldx,
                                                    ((int64_t)(tokens - 1) * p.ldx + p.K) * (int64_t)sizeof(X));
        auto x_at = [&](int t, int step, int i) {
            const int k = k_of(step, i), row = min(t * 16 + low, tokens - 1);
            if constexpr (BUF) {
                Raw8<X> r;
                const uint32_t at = k < p.K && step < steps ? ((uint32_t)row * (uint32_t)p.ldx + k) * (uint32_t)sizeof(X) : 0xffffff00u;
#pragma unroll
                for (int c = 0; c < (int)sizeof(X) / 2; ++c) r.v[c] = __builtin_amdgcn_raw_buffer_load_b128(rx, at + 16 * c, 0, 0);
                return r;
            } else {
                return raw8((const X *)p.x + (t0 + row) * p.ldx + k, step < steps ? p.K - k : 0);
            }
        };
        auto fetch = [&](int step, Step &f) {
            const uint32_t g0 = (uint32_t)(min(step, steps - 1) * kGroups);
            if constexpr (!SIGNED) {   // first, so that waits for what follows count the same either way
#pragma unroll
                for (int a = 0; a < NR; ++a) {
                    const uint32_t g = srow[a % MT] + g0;
                    if (kGroups == 1) {
                        f.z[a] = __builtin_amdgcn_raw_buffer_load_b8(rz[a / MT], g, 0, 0);
                    } else if (whole_zeros) {
                        f.z[a] = kGroups == 4 ? __builtin_amdgcn_raw_buffer_load_b32(rz[a / MT], g, 0, 0)
                                              : __builtin_amdgcn_raw_buffer_load_b16(rz[a / MT], g, 0, 0);
                    } else {
                        f.z[a] = 0;
#pragma unroll
                        for (int c = 0; c < kGroups; ++c)
                            f.z[a] |= (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(rz[a / MT], g + c, 0, 0) << (8 * c);
                    }
                }
            }
#pragma unroll
            for (int a = 0; a < NR; ++a) {
                const uint32_t g = srow[a % MT] + g0;
                const uint32_t at = step < steps ? (qrow[a % MT] + step * 16 + quarter * 4) * 4 : 0xffffff00u;
                f.w[a] = __builtin_amdgcn_raw_buffer_load_b128(rq[a / MT], at, 0, 0);
                // a step's scales together; those behind the row's last group are not used below
                if constexpr (kGroups == 4) {
                    const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(rs[a / MT], g * 4, 0, 0);
#pragma unroll
                    for (int c = 0; c < 4; ++c) f.s[a][c] = __uint_as_float(v[c]);
                } else if constexpr (kGroups == 2) {
                    const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(rs[a / MT], g * 4, 0, 0);
                    f.s[a][0] = __uint_as_float(v[0]), f.s[a][1] = __uint_as_float(v[1]);
                } else {
                    f.s[a][0] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs[a / MT], g * 4, 0, 0));
                }
            }
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) f.x[t][i] = x_at(t, step, i);
        };
        auto use = [&](const Step &f, int step) {
            u32x4 words_of[NR];
#pragma unroll
            for (int a = 0; a < NR; ++a) by_instruction(words_of[a] = f.w[a]);
#pragma unroll
            for (int c = 0; c < kGroups; ++c) {
                f32x4 part[NR][TT] = {};
                ZeroPoint z[NR];
#pragma unroll
                for (int a = 0; a < NR; ++a) z[a] = zero_point<SIGNED>(SIGNED ? 0u : (f.z[a] >> (8 * c)) & 255u);
#pragma unroll
                for (int b = 0; b < PER; ++b) {
                    const int i = c * PER + b;
                    u32x4 x[TT][kPieces<X>];
#pragma unroll
                    for (int t = 0; t < TT; ++t) {
                        Raw8<X> r = f.x[t][i];
                        if (BUF && step * 128 + 128 > p.K) clear_behind(r, p.K - k_of(step, i));
                        x_operand_paired(r, x[t]);
                    }
#pragma unroll
                    for (int a = 0; a < NR; ++a) {
                        const u32x4 v = whole_operand<H, SIGNED>(words_of[a][i], z[a]);
#pragma unroll
                        for (int t = 0; t < TT; ++t)
#pragma unroll
                            for (int j = 0; j < kPieces<X>; ++j) part[a][t] = mfma<H>(x[t][j], v, part[a][t]);
                    }
                }
                if (kGroups > 1 && step * kGroups + c >= groups) break;   // behind the row's last group
#pragma unroll
                for (int a = 0; a < NR; ++a)
#pragma unroll
                    for (int t = 0; t < TT; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[a][t][r] = fmaf(f.s[a][c], part[a][t][r], acc[a][t][r]);
            }
        };
        Step f0, f1;
        fetch(wave, f0);
        int step = wave;
        for (; step + kNarrowWaves < steps; step += 2 * kNarrowWaves) {
            fetch(step + kNarrowWaves, f1);
            use(f0, step);
            fetch(step + 2 * kNarrowWaves, f0);
            use(f1, step + kNarrowWaves);
        }
        if (step < steps) use(f0, step);
    };
    if (buffered) body(std::true_type{});
    else body(std::false_type{});

    // the waves' sums meet in LDS and are added in the waves' order
#pragma unroll
    for (int a = 0; a < NR; ++a)
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) meet[(wave * kPart + (a * TT + t) * 4 + r) * 64 + lane] = acc[a][t][r];
    __syncthreads();
    for (int n = threadIdx.x; n < kTokens * kRows; n += 64 * kNarrowWaves) {
        const int t = n / kRows, m = n % kRows;
        if (t >= tokens || m >= rows) continue;
        // lane (quarter, low) held tokens 4 quarter + r of row `low` of a set
        const int at = ((m / 16 * TT + t / 16) * 4 + t % 4) * 64 + t % 16 / 4 * 16 + m % 16;
        float v[NW] = {};
#pragma unroll
        for (int a = 0; a < NW; ++a)
#pragma unroll
            for (int w = 0; w < kNarrowWaves; ++w) v[a] += meet[(w * kPart + a * MT * TT * 4) * 64 + at];
        float out = v[0];
        if constexpr (NW > 1) {
            float da;
            activation(p.act, v[0], out, da);
            out *= v[1];
        }
        ((X *)p.y)[(t0 + t) * p.ldy + m0 + m] = (X)out;
    }
}

// Launches the kernel: 16 tokens a workgroup, or 32; 16 rows of W, or, where those are two workgroups and more for each
// CU, 32, which read x half as often (16 x 8192 x 8192, unsigned groups of 64: 29.0 us with 16 rows, 22.0 with 32;
// 16 x 4096 x 4096: 9.7 and 12.9).  The gated block's two matrices share x already: 32 rows of each are slower always.
template <class X, bool SIGNED, int NW>
int launch_narrow(const GroupProduct &p, int words, int groups, hipStream_t s) {
    const int tt = p.T <= 16 ? 1 : 2;
    const int64_t tblocks = ((int64_t)p.T + 16 * tt - 1) / (16 * tt);
    const int mt = NW == 1 && tblocks * (((int64_t)p.M + 15) / 16) >= 512 ? 2 : 1;
    const int64_t blocks = tblocks * (((int64_t)p.M + 16 * mt - 1) / (16 * mt));
    if (const int st = check_blocks(blocks, 64 * kNarrowWaves, "group product")) return st;
    const bool buffered = within_buffer(p.x, sizeof(X), std::min<int64_t>(p.T, 32), p.ldx, p.K);
    // a step's zero points (4 bytes for groups of 32, 2 for groups of 64) in one access
    bool whole_zeros = groups % (128 / p.group) == 0;
    for (int a = 0; a < NW; ++a) whole_zeros = whole_zeros && (uintptr_t)p.w[a].zero % (128 / p.group) == 0;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(64 * kNarrowWaves), 0, s, p, words, groups, buffered,
                           whole_zeros);
    };
    auto with_group = [&](auto per) {
        constexpr int PER = decltype(per)::value;
        if constexpr (NW == 1)
            if (mt == 2) {
                tt == 1 ? go(group_narrow_kernel<X, SIGNED, PER, 1, NW, 2>) : go(group_narrow_kernel<X, SIGNED, PER, 2, NW, 2>);
                return;
            }
        tt == 1 ? go(group_narrow_kernel<X, SIGNED, PER, 1, NW, 1>) : go(group_narrow_kernel<X, SIGNED, PER, 2, NW, 1>);
    };
    if (p.group == 32) with_group(std::integral_constant<int, 1>{});
    else if (p.group == 64) with_group(std::integral_constant<int, 2>{});
    else with_group(std::integral_constant<int, 4>{});
    return check_launch("group product");
}

}  // namespace samd
