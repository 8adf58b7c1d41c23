// Products of one or two tokens with 4-bit group-scaled weights (the decoding step of a language
// model): y[t][m] = sum_g s[m][g] sum_{k in g} (u[m][k] - z[m][g]) x[t][k], u the field 0..15
// (a signed field with its sign bit flipped, its zero point then being 8).
//
// Bound by reading the weights, half a byte a value, so at the card's 5.2 TB/s there are three to
// four lane operations for each value.  A lane takes 32 consecutive values of a row, 16 bytes, which
// one scale covers whatever the group, and keeps every operation whole-word:
//   16-bit types  (16 + u) / 16 is a 16-bit float whose top four mantissa bits are u, so two values
//                 become two floats by one shift and one and-xor, and a two-way dot product adds both:
//                 sum x (u - z) = 16 sum x (16 + u)/16 - (16 + z) sum x, sum x once for all rows
//   f32           fields to floats by byte conversions, one multiply-add each
// The offset of 16 costs the 32-bit sum two bits at most; the products themselves are exact.
//
// Measured (graph of calls, bf16, one token): 16384 x 8192 weights 14.8 us, 4.8 TB/s of weights, scales and x;
// 4096 x 4096 4.6 us, of which a launch that does next to nothing (512 x 512) is 3.5.
//
// A wave computes R rows of each matrix along all of K, 2048 values a step, the next step's weights
// requested before this one's are used; x waits in LDS in the order in which fields come out of a
// word, [token][step][word of the lane][lane], so its 16-byte reads meet no bank twice.
#pragma once

#include "group_device.hpp"

namespace samd {

constexpr int kVecWaves = 4;          // waves of a workgroup
constexpr int kVecStep = 2048;        // values of a row per step: 64 lanes x 32
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

template <class X>
__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) {
    if constexpr (std::is_same_v<X, half_t>)
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(half2_t, a), __builtin_bit_cast(half2_t, b), c, false);
    else
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf162_t, a), __builtin_bit_cast(bf162_t, b), c, false);
}

// Fields i and i + 4 of a word as the floats (16 + u) / 16 of the type; `one` is two floats 1, with their top
// mantissa bit set where the fields are signed (which flips the field's sign bit: u is the value plus 8).
template <class X, int I>
__device__ __forceinline__ uint32_t field_pair(uint32_t w, uint32_t one) {
    constexpr int kAt = std::is_same_v<X, half_t> ? 6 : 3;   // lowest of the top four mantissa bits
    constexpr int kShift = kAt - 4 * I;
    const uint32_t t = kShift >= 0 ? w << (kShift >= 0 ? kShift : 0) : w >> (kShift < 0 ? -kShift : 0);
    return (t & (0x000f000fu << kAt)) ^ one;
}

template <class X, bool SIGNED, int T, int NW, int R>
__global__ __launch_bounds__(64 * kVecWaves) void group_vector_kernel(GroupProduct p, int words, int groups, int gshift,
                                                                      int steps, int held) {
    constexpr bool kWide = sizeof(X) == 4;
    constexpr int kParts = kWide ? 8 : 4;          // 16-byte parts of a lane's 32 values of x
    extern __shared__ u32x4 xs[];                  // [T][held][kParts][64], then float sums [T][held][64]
    float *const sums = (float *)(xs + T * held * kParts * 64);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t m0 = ((int64_t)blockIdx.x * kVecWaves + wave) * R;
    constexpr uint32_t one = std::is_same_v<X, half_t> ? (SIGNED ? 0x3e003e00u : 0x3c003c00u)
                                                       : (SIGNED ? 0x3fc03fc0u : 0x3f803f80u);

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
                if (!SIGNED) f.z[a][r] = __builtin_amdgcn_raw_buffer_load_b8(rz[a], g + (uint32_t)r * (uint32_t)groups, 0, 0);
            }
    };
    float acc[NW][R][T] = {};
    // one step: 32 values of every row in this lane
    auto use = [&](const Step &f, int s) {
        float part[NW][R][T] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u32x4 x[T][kParts / 4];
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int c = 0; c < kParts / 4; ++c) x[t][c] = xs[((t * held + s) * kParts + i * (kParts / 4) + c) * 64 + lane];
#pragma unroll
            for (int a = 0; a < NW; ++a)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    if constexpr (kWide) {
                        const uint32_t w = SIGNED ? f.w[a][r][i] ^ 0x88888888u : f.w[a][r][i];
                        const uint32_t lo = as_is(w & 0x0f0f0f0fu), hi = as_is((w >> 4) & 0x0f0f0f0fu);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float e = (float)((lo >> (8 * j)) & 255u), o = (float)((hi >> (8 * j)) & 255u);
#pragma unroll
                            for (int t = 0; t < T; ++t) {
                                part[a][r][t] = fmaf(e, __uint_as_float(x[t][0][j]), part[a][r][t]);
                                part[a][r][t] = fmaf(o, __uint_as_float(x[t][kParts / 4 - 1][j]), part[a][r][t]);
                            }
                        }
                    } else {
                        const uint32_t w = f.w[a][r][i];
                        const uint32_t v[4] = {field_pair<X, 0>(w, one), field_pair<X, 1>(w, one), field_pair<X, 2>(w, one),
                                               field_pair<X, 3>(w, one)};
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int t = 0; t < T; ++t) part[a][r][t] = dot2<X>(v[j], x[t][0][j], part[a][r][t]);
                    }
                }
        }
        float sum[T];
#pragma unroll
        for (int t = 0; t < T; ++t) sum[t] = sums[(t * held + s) * 64 + lane];
#pragma unroll
        for (int a = 0; a < NW; ++a)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                // kWide: s (part - z sum); else 16 s (part - (1 + z/16) sum), both factors exact
                const float z = SIGNED ? 8.0f : (float)f.z[a][r];
                const float zz = kWide ? -z : fmaf(z, -0.0625f, -1.0f), s2 = kWide ? f.s[a][r] : 16.0f * f.s[a][r];
#pragma unroll
                for (int t = 0; t < T; ++t) acc[a][r][t] = fmaf(s2, fmaf(zz, sum[t], part[a][r][t]), acc[a][r][t]);
            }
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
            u32x4 *to = xs + (at * kParts + (j & 3) * (kParts / 4)) * 64 + to_lane;
            if constexpr (kWide) {   // fields come out of a word as 0, 2, 4, 6 and 1, 3, 5, 7
                to[0] = __builtin_bit_cast(u32x4, f32x4{v[0], v[2], v[4], v[6]});
                to[64] = __builtin_bit_cast(u32x4, f32x4{v[1], v[3], v[5], v[7]});
            } else {
                const Eight<X> h = {{(X)v[0], (X)v[4], (X)v[1], (X)v[5], (X)v[2], (X)v[6], (X)v[3], (X)v[7]}};
                to[0] = __builtin_bit_cast(u32x4, h);
            }
            // four neighbouring threads hold a lane's 32 values
            float sum = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
            sum += lane_swap<0xb1>(sum);
            sum += lane_swap<0x4e>(sum);
            if ((j & 3) == 0) sums[at * 64 + to_lane] = sum;
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
// 9.5 with two; 16384 x 8192: 17.7 and 14.8).
template <class X, bool SIGNED, int NW>
int launch_vector(const GroupProduct &p, int words, int groups, int gshift, hipStream_t s) {
    const int steps = (words + 255) / 256;
    const bool one = p.M <= 2048;
    const int rows = kVecWaves * (one ? 1 : 2);
    const int64_t blocks = ((int64_t)p.M + rows - 1) / rows;
    if (const int st = check_blocks(blocks, 64 * kVecWaves, "group product")) return st;
    const dim3 grid((uint32_t)blocks);
    auto go = [&](auto kernel, int tokens) {
        const int step_bytes = tokens * (kVecStep * (int)sizeof(X) + 256);
        const int held = std::min(steps, std::max(2, kVecLds / step_bytes & ~1));
        hipLaunchKernelGGL(kernel, grid, dim3(64 * kVecWaves), held * step_bytes, s, p, words, groups, gshift, steps, held);
    };
    if (p.T == 1) one ? go(group_vector_kernel<X, SIGNED, 1, NW, 1>, 1) : go(group_vector_kernel<X, SIGNED, 1, NW, 2>, 1);
    else one ? go(group_vector_kernel<X, SIGNED, 2, NW, 1>, 2) : go(group_vector_kernel<X, SIGNED, 2, NW, 2>, 2);
    return check_launch("group product");
}

}  // namespace samd
