// Products of one or two tokens with 4-bit group-scaled weights (the decoding step of a language
// model): y[t][m] = sum_g s[m][g] sum_{k in g} (u[m][k] - z[m][g]) x[t][k], u the field 0..15
// (a signed field with its sign bit flipped, its zero point then being 8).
//
// Bound by reading the weights, half a byte a value, so at the card's 5.2 TB/s there are three to
// four lane operations for each value.  A lane takes 32 consecutive values of a row, 16 bytes, which
// one scale covers whatever the group, and keeps every operation whole-word: two fields at a time become the 16-bit floats
// u - z, exactly (whole_pairs: 9 operations for 8 of them), and a multiply-add of mixed types adds one, times a 32-bit x,
// to a 32-bit sum.  A weight equal to its zero point adds nothing, and each product is rounded once, with its sum.
//
// Measured (graph of calls, one token): 16384 x 8192 weights in unsigned groups of 128 bf16 17.0 us (4.2 TB/s of weights,
// scales and x), f16 17.5, f32 16.8; 4096 x 4096 4.7 us, of which a launch that does next to nothing (512 x 512) is 3.6.
//
// A wave computes R rows of each matrix along all of K, 2048 values a step, the next step's weights
// requested before this one's are used; x waits in LDS as 32-bit floats, a lane's halves of words apart,
// [token][step][half of a word][lane], so its 16-byte reads meet no bank twice.
#pragma once

#include "group_device.hpp"

namespace samd {

constexpr int kVecWaves = 4;          // waves of a workgroup
constexpr int kVecStep = 2048;        // values of a row per step: 64 lanes x 32
constexpr int kVecParts = 8;          // 16-byte parts of a lane's 32 values of x
constexpr int kVecLds = 32768;        // bytes of x held at once

// v of the lane that a data-parallel control names, within rows of 16 lanes.
template <int CTRL>
__device__ __forceinline__ float lane_swap(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// Sum over a wave, in every lane, in a fixed order: within 16 lanes by data-parallel primitives,
// then the four rows of 16.
__device__ __forceinline__ float wave_sum(float v) {
    v += lane_swap<0xb1>(v);    // lane ^ 1
    v += lane_swap<0x4e>(v);    // lane ^ 2
    v += lane_swap<0x141>(v);   // mirrored within 8
    v += lane_swap<0x140>(v);   // mirrored within 16
    const float a = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 0));
    const float b = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 16));
    const float c = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 32));
    const float d = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 48));
    return (a + b) + (c + d);
}

template <class X, bool SIGNED, int T, int NW, int R>
__global__ __launch_bounds__(64 * kVecWaves) void group_vector_kernel(GroupProduct p, int words, int groups, int gshift,
                                                                      int steps, int held) {
    extern __shared__ f32x4 xs[];                  // [T][held][kVecParts][64]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t m0 = ((int64_t)blockIdx.x * kVecWaves + wave) * R;

    // The wave's rows through buffer descriptors that end with its last row (or W's): what a lane asks for
    // behind the end reads as 0, and what it gets from the next row meets an x of 0.
    const int64_t first = min(m0, (int64_t)p.M - 1);
    const int rows = (int)min((int64_t)R, p.M - first);
    __amdgpu_buffer_rsrc_t rq[NW], rs[NW], rz[NW];
#pragma unroll
    for (int a = 0; a < NW; ++a) {
        rq[a] = buffer_of(p.w[a].q + first * words, (int64_t)rows * words * 4);
        rs[a] = buffer_of(p.w[a].scale + first * groups, (int64_t)rows * groups * 4);
        rz[a] = byte_buffer_of(p.w[a].zero + first * groups, SIGNED ? 0 : (int64_t)rows * groups);
    }
    struct Step {
        u32x4 w[NW][R];
        float s[NW][R];
        uint32_t z[NW][R];
    };
    auto fetch = [&](int step, Step &f) {
        // always requested, so that the wait for a step's weights leaves the next step's in flight; a step
        // behind the last is asked for behind the buffer's end, which reads no memory
        const uint32_t at = step < steps ? (uint32_t)(step * 1024 + lane * 16) : 0xc0000000u;
        const uint32_t g = (uint32_t)min((step * kVecStep + lane * 32) >> gshift, groups - 1);
#pragma unroll
        for (int a = 0; a < NW; ++a)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                f.w[a][r] = __builtin_amdgcn_raw_buffer_load_b128(rq[a], at + (uint32_t)r * (uint32_t)words * 4u, 0, 0);
                f.s[a][r] =
                    __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs[a], (g + (uint32_t)r * (uint32_t)groups) * 4, 0, 0));
                f.z[a][r] = SIGNED ? 0u : __builtin_amdgcn_raw_buffer_load_b8(rz[a], g + (uint32_t)r * (uint32_t)groups, 0, 0);
            }
    };
    float acc[NW][R][T] = {};
    // one step: 32 values of every row in this lane
    auto use = [&](const Step &f, int s) {
        float part[NW][R][T] = {};
        ZeroPoint z[NW][R];
#pragma unroll
        for (int a = 0; a < NW; ++a)
#pragma unroll
            for (int r = 0; r < R; ++r) z[a][r] = zero_point<SIGNED>(f.z[a][r]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4 x[T][2];   // values 0 .. 3 and 4 .. 7 of a word
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int c = 0; c < 2; ++c) x[t][c] = xs[((t * held + s) * kVecParts + i * 2 + c) * 64 + lane];
#pragma unroll
            for (int a = 0; a < NW; ++a)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    half2_t v[4];
                    whole_pairs<SIGNED>(f.w[a][r][i], z[a][r], v);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int t = 0; t < T; ++t) {
                            part[a][r][t] = fmaf((float)v[j][0], x[t][0][j], part[a][r][t]);
                            part[a][r][t] = fmaf((float)v[j][1], x[t][1][j], part[a][r][t]);
                        }
                }
        }
#pragma unroll
        for (int a = 0; a < NW; ++a)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int t = 0; t < T; ++t) acc[a][r][t] = fmaf(f.s[a][r], part[a][r][t], acc[a][r][t]);
    };

    Step f0, f1;
    fetch(0, f0);
    for (int s0 = 0; s0 < steps; s0 += held) {   // held is even, or all of K: f0 is always the first step's
        const int here = min(held, steps - s0);
        if (s0) __syncthreads();
        for (int i = threadIdx.x; i < here * 256 * T; i += 64 * kVecWaves) {
            const int t = i / (here * 256), j = i - t * (here * 256);   // the 8 values of word j
            const int64_t k0 = ((int64_t)s0 * 256 + j) * 8;
            float v[8] = {};
            if (t < p.T && k0 < p.K) load8((const X *)p.x + (int64_t)t * p.ldx + k0, (int)min((int64_t)8, p.K - k0), v);
            const int at = t * held + (j >> 8), to_lane = (j & 255) >> 2;
            f32x4 *to = xs + (at * kVecParts + (j & 3) * 2) * 64 + to_lane;
            to[0] = f32x4{v[0], v[1], v[2], v[3]};
            to[64] = f32x4{v[4], v[5], v[6], v[7]};
        }
        __syncthreads();
        // no way out between the two halves: the compiler would move the request behind it
        for (int s = 0; s + 2 <= here; s += 2) {
            fetch(s0 + s + 1, f1);
            use(f0, s);
            fetch(s0 + s + 2, f0);
            use(f1, s + 1);
        }
        if (here & 1) use(f0, here - 1);   // K's last step
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < T; ++t) {
            float out = wave_sum(acc[0][r][t]);
            if constexpr (NW > 1) {
                float a, da;
                activation(p.act, out, a, da);
                out = a * wave_sum(acc[NW - 1][r][t]);
            }
            if (lane == 0 && m0 + r < p.M && t < p.T) ((X *)p.y)[(int64_t)t * p.ldy + m0 + r] = (X)out;
        }
}

// Launches the kernel for p.T tokens (1 or 2).  Two rows a wave, so that x is read from LDS half as
// often, unless that leaves CUs without a workgroup (1024 x 16384 weights: 7.4 us with one row a wave,
// 9.6 with two; 16384 x 8192: 21.7 and 17.2).
template <class X, bool SIGNED, int NW>
int launch_vector(const GroupProduct &p, int words, int groups, int gshift, hipStream_t s) {
    const int steps = (words + 255) / 256;
    const bool one = p.M <= 2048;
    const int rows = kVecWaves * (one ? 1 : 2);
    const int64_t blocks = ((int64_t)p.M + rows - 1) / rows;
    if (const int st = check_blocks(blocks, 64 * kVecWaves, "group product")) return st;
    const dim3 grid((uint32_t)blocks);
    auto go = [&](auto kernel, int tokens) {
        const int step_bytes = tokens * kVecStep * (int)sizeof(float);
        const int held = std::min(steps, std::max(2, kVecLds / step_bytes & ~1));
        hipLaunchKernelGGL(kernel, grid, dim3(64 * kVecWaves), held * step_bytes, s, p, words, groups, gshift, steps, held);
    };
    if (p.T == 1) one ? go(group_vector_kernel<X, SIGNED, 1, NW, 1>, 1) : go(group_vector_kernel<X, SIGNED, 1, NW, 2>, 1);
    else one ? go(group_vector_kernel<X, SIGNED, 2, NW, 1>, 2) : go(group_vector_kernel<X, SIGNED, 2, NW, 2>, 2);
    return check_launch("group product");
}

}  // namespace samd
