// Products of many tokens with 4-bit group-scaled weights on the matrix cores, and the gated block on two of them.
//
// A field minus its zero point is a whole number of -15..15, exact as a 16-bit float, so it is multiplied
// exactly and scaled once for each group and output, in 32-bit floats: no weight is ever rounded.  32-bit
// activations enter as three bf16 pieces (three instructions a product).
//
// A workgroup computes 16 WT TW tokens x 16 WM MW rows of W with TW x MW waves for each of KS slices of K, a
// wave 16 WT x 16 WM: large tiles where there are many tokens, slices where there are too few to fill the card.  Steps of 64
// values: x (copied) and the fields (decoded once for the workgroup) go through LDS, two buffers, the next
// step's loads in flight during this step's products.
// W is the first operand: a lane then ends with 4 consecutive rows of W for a token, which are stored together
// and are one word of the gated block's stored projections.
//
// Measured (graph of calls, 4096 x 4096 weights): 2048 tokens bf16 or f16 85 us with signed groups of 128 (807 TFLOP/s of
// the 1150 that a large library product reaches), 106 us with unsigned groups of 32 (twice the scaling and its sums),
// f32 225 us; 256 tokens 24 us, 64 tokens 15 us.  In the largest tile the phases that fetch bound it (operands
// out of LDS, decoding, writing the next step: 78 us were the products left out, the products alone 59), which is why
// two groups of waves alternate; few tokens are bound by a workgroup's chain of steps.
#pragma once

#include "group_device.hpp"

namespace samd {

// A lambda that is part of its kernel however often it is called: its arrays have to stay in registers.
#define SAMD_INLINE __attribute__((always_inline))

constexpr int kGemmStep = 64;

// Index of 16-byte part `c` (0..7) of row `r` in a buffer of rows of 64 16-bit values.  Of 16 rows, 0..7 lie in the lower
// halves of 256 bytes (all banks), 8..15 in the upper ones, their parts exchanged by r % 8: neither the 16 rows that an
// operand's lanes read at one c, nor 8 parts of two rows that are 8 apart, meet a bank twice.
__device__ __forceinline__ int part_at(int r, int c) { return ((r & ~15) + (r & 7) * 2 + (r >> 3 & 1)) * 8 + (c ^ (r & 7)); }

// 8 fields of a word minus z as 16-bit floats in order (z + 8 for signed fields, whose sign bits are flipped).
template <class H>
__device__ __forceinline__ u32x4 whole_values(uint32_t w, int z) {
    if constexpr (std::is_same_v<H, half_t>) {
        // 1024 + u in a half's lowest bits, two fields at a time; minus 1024 + z is exact
        const half_t off = (half_t)(1024 + z);
        const half2_t offs = {off, off};
        uint32_t t[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            t[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, (w >> (4 * i) & 0x000f000fu) | 0x64006400u) - offs);
        return u32x4{__builtin_amdgcn_perm(t[1], t[0], 0x05040100u), __builtin_amdgcn_perm(t[3], t[2], 0x05040100u),
                     __builtin_amdgcn_perm(t[1], t[0], 0x07060302u), __builtin_amdgcn_perm(t[3], t[2], 0x07060302u)};
    } else {
        const uint32_t lo = as_is(w & 0x0f0f0f0fu), hi = as_is((w >> 4) & 0x0f0f0f0fu);
        const float zf = (float)z;
        u32x4 out;
#pragma unroll
        for (int j = 0; j < 4; ++j) {   // whole floats of at most 4 bits: their upper halves are the bf16
            const float e = (float)((lo >> (8 * j)) & 255u) - zf, o = (float)((hi >> (8 * j)) & 255u) - zf;
            out[j] = __builtin_amdgcn_perm(__float_as_uint(o), __float_as_uint(e), 0x07060302u);
        }
        return out;
    }
}

// Workgroup b of n as one of n tiles, so that neighbouring tiles run on one XCD (workgroups go to the eight in turn)
// and share its L2.
__device__ __forceinline__ uint32_t tile_of(uint32_t b, uint32_t n) {
    const uint32_t xcd = b % kNumXcd, per = n / kNumXcd, more = n % kNumXcd;
    return xcd * per + min(xcd, more) + b / kNumXcd;
}

// Rows of a float matrix (from row r0 on, `rows` of them in range) on their way into LDS as matrix operands:
// ROWS x 64 values a step.
// BUF: the rows are on 4 bytes and within 4 GB, and are read through one descriptor; else value by value.
template <class X, int ROWS, int THREADS, bool BUF>
struct TokenTile {
    static constexpr int kEach = ROWS * 8 / THREADS;   // 8-value parts of a thread
    Raw8<X> raw[kEach];

    // What stands behind a row's end comes along and is cleared by store().
    __device__ __forceinline__ void load(const __amdgpu_buffer_rsrc_t &rx, const X *x, int64_t ld, int rows, int cols, int step, int tid) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int row = min(e * (THREADS / 8) + tid / 8, rows - 1), k = tid % 8 * 8;
            if constexpr (BUF) {
                const uint32_t at = ((uint32_t)row * (uint32_t)ld + k) * (uint32_t)sizeof(X) + step * (kGemmStep * (int)sizeof(X));
#pragma unroll
                for (int c = 0; c < (int)sizeof(X) / 2; ++c)
                    raw[e].v[c] = __builtin_amdgcn_raw_buffer_load_b128(rx, at + 16 * c, 0, 0);
            } else {
                raw[e] = raw8(x + row * ld + step * kGemmStep + k, cols - step * kGemmStep - k);
            }
        }
    }

    // RAGGED: the step may reach behind the rows' end.  convert(): 8 values as P matrix operands.
    template <bool RAGGED, int P, class F>
    __device__ __forceinline__ void store(u32x4 (&to)[P][ROWS * 8], int cols, int step, int tid, F &&convert) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int id = e * THREADS + tid;
            if (RAGGED) clear_behind(raw[e], cols - (step * kGemmStep + id % 8 * 8));
            u32x4 piece[P];
            convert(raw[e], piece);
#pragma unroll
            for (int j = 0; j < P; ++j) to[j][part_at(id / 8, id % 8)] = piece[j];
        }
    }
};

// 4 neighbouring results of a row, `n` of them in range.
template <class X>
__device__ __forceinline__ void store4(X *p, int n, const float (&v)[4]) {
    struct {
        X v[4];
    } t;
#pragma unroll
    for (int i = 0; i < 4; ++i) t.v[i] = (X)v[i];
    if (n >= 4) {
        if constexpr (sizeof(X) == 4) *(u32x4_at4 *)p = __builtin_bit_cast(u32x4, t);
        else *(u32x2_at2 *)p = __builtin_bit_cast(u32x2, t);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = t.v[i];
    }
}

template <class X, bool BUF, int PER, int NW, int WT, int WM, int TW, int MW, int KS>
__global__ __launch_bounds__(64 * TW * MW * KS) void group_gemm_kernel(GroupProduct p, int words, int groups, int tblocks) {
    using H = std::conditional_t<std::is_same_v<X, half_t>, half_t, bf16_t>;
    constexpr int P = kPieces<X>, THREADS = 64 * TW * MW;
    constexpr int BT = 16 * WT * TW, BM = 16 * WM * MW;      // tokens and rows of W of a workgroup
    constexpr int OM = BM / NW;                               // rows of the result
    constexpr int WPT = BM * 8 / THREADS;                     // words of a thread and step
    constexpr int TPR = 8 / WPT;                              // threads of a row
    constexpr int SG = PER == 1 ? 2 : 1;                      // groups of a step
    static_assert(64 / TPR <= 16 * WM / NW || NW == 1, "a wave decodes rows of one matrix");
    struct Buffers {   // of one slice of K
        u32x4 x[2][P][BT * 8], w[2][BM * 8];
        float s[2][SG * BM];
    };
    static_assert((KS - 1) * BT * BM * 4 <= (int)sizeof(Buffers) * KS, "the slices' sums meet in the buffers");
    __shared__ Buffers all[KS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % (TW * MW);
    const int slice = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / (TW * MW), tid = threadIdx.x - slice * THREADS;
    auto &xs = all[slice].x;
    auto &ws = all[slice].w;
    auto &ss = all[slice].s;
    const int quarter = lane >> 4, low = lane & 15, tw = wave % TW, mw = wave / TW;
    const uint32_t tile = tile_of(blockIdx.x, gridDim.x);
    const int64_t t0 = (int64_t)(tile % tblocks) * BT, m0 = (int64_t)(tile / tblocks) * OM;
    const int tokens = (int)min((int64_t)BT, p.T - t0), rows = (int)min((int64_t)OM, p.M - m0);
    const int steps = (p.K + kGemmStep - 1) / kGemmStep;

    const X *x = (const X *)p.x + t0 * p.ldx;
    const __amdgpu_buffer_rsrc_t rx = buffer_of(x, ((int64_t)(tokens - 1) * p.ldx + p.K) * (int64_t)sizeof(X));
    // Row r of the buffer: a wave's 16 WM rows are first its rows of W[0], then those of W[1].  A wave decodes rows of one.
    auto matrix_of = [](int r) { return NW == 1 ? 0 : r % (16 * WM) / (8 * WM); };
    auto result_row = [](int r) { return NW == 1 ? r : r / (16 * WM) * (8 * WM) + r % (8 * WM); };
    const int wrow = tid / TPR, part = tid % TPR * WPT;
    const int a = __builtin_amdgcn_readfirstlane(matrix_of(wrow));
    const int row = result_row(wrow);
    const bool has_zero = p.w[0].zero != nullptr;
    const uint32_t flip = has_zero ? 0u : 0x88888888u;
    const __amdgpu_buffer_rsrc_t rq = buffer_of(p.w[a].q + m0 * words, (int64_t)rows * words * 4);
    const __amdgpu_buffer_rsrc_t rz = byte_buffer_of(p.w[a].zero + m0 * groups, has_zero ? (int64_t)rows * groups : 0);
    const uint32_t qrow = (uint32_t)row * (uint32_t)words, zrow = (uint32_t)row * (uint32_t)groups;
    // scales: a thread loads those of row tid % BM of the buffer
    static_assert(THREADS % BM == 0, "a thread loads the scales of one row");
    const int srow = result_row(tid % BM);
    const bool scales = srow < rows;
    const float *const sp = p.w[matrix_of(tid % BM)].scale + (m0 + (scales ? srow : 0)) * groups;

    struct Step {
        TokenTile<X, BT, THREADS, BUF> x;
        uint32_t q[WPT], z;
        float s[SG];
    };
    auto load = [&](Step &f, int step) SAMD_INLINE {
        step = __builtin_amdgcn_readfirstlane(step);
        asm("" : "+s"(step));   // addresses from one scalar each turn, not a register carried for each of them
        f.x.load(rx, x, p.ldx, tokens, p.K, step, tid);
        // steps behind the last get the next row's words, or zeros, for an x of zeros
        const uint32_t at = (row < rows ? (qrow + part) * 4 : 0xc0000000u) + step * 32;
        if constexpr (WPT == 4) {
            const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(rq, at, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) f.q[i] = v[i];
        } else {
            const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(rq, at, 0, 0);
            f.q[0] = v[0], f.q[1] = v[1];
        }
        // a thread's words lie in one group
        f.z = __builtin_amdgcn_raw_buffer_load_b8(rz, zrow + (PER == 1 ? part / 4 : 0) + step * kGemmStep / (32 * PER), 0, 0);
#pragma unroll
        for (int c = 0; c < SG; ++c) f.s[c] = sp[min(step * kGemmStep / (32 * PER) + c, groups - 1)];
    };
    auto store = [&](auto ragged, Step &f, int step, int buf) SAMD_INLINE {
        f.x.template store<decltype(ragged)::value>(xs[buf], p.K, step, tid, [](const Raw8<X> &r, u32x4(&o)[P]) { x_operand(r, o); });
#pragma unroll
        for (int i = 0; i < WPT; ++i)
            ws[buf][part_at(wrow, part + i)] = whole_values<H>(f.q[i] ^ flip, has_zero ? (int)f.z : 8);
#pragma unroll
        for (int c = 0; c < SG; ++c)   // threads of one row write one value
            ss[buf][c * BM + tid % BM] = scales && step * kGemmStep / (32 * PER) + c < groups ? f.s[c] : 0.0f;
    };

    const int at[2] = {part_at(low, quarter), part_at(low, 4 + quarter)};   // the same in every 16 rows
    f32x4 acc[WM][WT] = {};
    u32x4 av[2][WM];
    f32x4 scale[SG][WM];
    Step f;
    auto operands = [&](int buf) SAMD_INLINE {   // of W, and the scales
#pragma unroll
        for (int i = 0; i < WM; ++i) {
#pragma unroll
            for (int c = 0; c < 2; ++c) av[c][i] = ws[buf][(mw * WM + i) * 128 + at[c]];
#pragma unroll
            for (int c = 0; c < SG; ++c) scale[c][i] = *(const f32x4 *)&ss[buf][c * BM + (mw * WM + i) * 16 + quarter * 4];
        }
    };
    // A step's products with token tiles from .. to - 1.  The sums of a step (of each half where groups are 32) are
    // scaled at once: they live for a few instructions only.
    auto multiply = [&](auto &&x_of, int from, int to) SAMD_INLINE {
#pragma unroll
        for (int t = from; t < to; ++t) {
            f32x4 sum[SG][WM] = {};
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const u32x4 bv = x_of(c, j, t);
#pragma unroll
                    for (int i = 0; i < WM; ++i) sum[c % SG][i] = mfma<H>(av[c][i], bv, sum[c % SG][i]);
                }
#pragma unroll
            for (int c = 0; c < SG; ++c)
#pragma unroll
                for (int i = 0; i < WM; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][t][r] = fmaf(scale[c][i][r], sum[c][i][r], acc[i][t][r]);
        }
#pragma unroll
        for (int t = from; t < to; ++t)   // here, not behind the barrier, where the sums would still need registers
#pragma unroll
            for (int i = 0; i < WM; ++i) asm volatile("" : "+v"(acc[i][t]));
    };

    // Two steps a turn, so that the buffers are known.  The slices take turns in turn, all as many (steps behind
    // the last are zeros).
    const int turns = (steps + 2 * KS - 1) / (2 * KS);
    constexpr int NEXT = 2 * KS;
    int step = 2 * slice;
    load(f, step);
    store(std::true_type{}, f, step, 0);
    load(f, step + 1);
    __syncthreads();
    auto all_turns = [&](auto &&one) SAMD_INLINE {
        int turn = 0;
        for (; turn < turns && step + NEXT < p.K / kGemmStep; ++turn, step += NEXT) one(std::false_type{});
        for (; turn < turns; ++turn, step += NEXT) one(std::true_type{});
    };
    if constexpr (KS == 1 && TW * MW == 8) {
        // Eight waves, two on each SIMD: the second four run one phase behind the first, so that one wave of a
        // SIMD multiplies while the other fetches its operands and decodes.
        const bool behind = wave >= 4;
        u32x4 bv[2][P][WT];
        auto fetch = [&](auto ragged, int buf, int next) SAMD_INLINE {
            operands(buf);
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int j = 0; j < P; ++j)
#pragma unroll
                    for (int t = 0; t < WT; ++t) bv[c][j][t] = xs[buf][j][(tw * WT + t) * 128 + at[c]];
            store(ragged, f, next, buf ^ 1);
            load(f, next + 1);
            __syncthreads();
            __builtin_amdgcn_s_setprio(1);
            multiply([&](int c, int j, int t) SAMD_INLINE { return bv[c][j][t]; }, 0, WT);
            __builtin_amdgcn_s_setprio(0);
            __syncthreads();
        };
        if (behind) __syncthreads();
        all_turns([&](auto ragged) SAMD_INLINE {
            fetch(ragged, 0, step + 1);
            fetch(ragged, 1, step + 2);
        });
        if (!behind) __syncthreads();
    } else {
        // The next step's data goes into the other buffer between the products of the two halves of the tokens.
        auto both = [&](auto ragged, int buf, int next, int after) SAMD_INLINE {
            auto x_of = [&](int c, int j, int t) SAMD_INLINE { return xs[buf][j][(tw * WT + t) * 128 + at[c]]; };
            operands(buf);
            multiply(x_of, 0, WT / 2);
            store(ragged, f, next, buf ^ 1);
            multiply(x_of, WT / 2, WT);
            load(f, after);
            __syncthreads();
        };
        all_turns([&](auto ragged) SAMD_INLINE {
            both(ragged, 0, step + 1, step + NEXT);
            both(ragged, 1, step + NEXT, step + NEXT + 1);
        });
    }
    if constexpr (KS > 1) {   // the first slice's waves add the others' sums, in order
        f32x4 *meet = (f32x4 *)all;
        auto at_sum = [&](int from, int i, int t) { return ((((from - 1) * TW * MW + wave) * WM + i) * WT + t) * 64 + lane; };
        if (slice)
#pragma unroll
            for (int i = 0; i < WM; ++i)
#pragma unroll
                for (int t = 0; t < WT; ++t) meet[at_sum(slice, i, t)] = acc[i][t];
        __syncthreads();
        if (slice) return;
        for (int from = 1; from < KS; ++from)
#pragma unroll
            for (int i = 0; i < WM; ++i)
#pragma unroll
                for (int t = 0; t < WT; ++t) acc[i][t] += meet[at_sum(from, i, t)];
    }

#pragma unroll
    for (int t = 0; t < WT; ++t) {
        const int64_t token = t0 + (tw * WT + t) * 16 + low;
        const bool in = token < p.T;
        X *y = (X *)p.y + token * p.ldy;
        if constexpr (NW == 1) {
#pragma unroll
            for (int i = 0; i < WM; ++i) {
                const int64_t m = m0 + (mw * WM + i) * 16 + quarter * 4;
                const float v[4] = {acc[i][t][0], acc[i][t][1], acc[i][t][2], acc[i][t][3]};
                if (in) store4(y + m, (int)min((int64_t)4, p.M - m), v);
            }
        } else {
            static_assert(NW == 1 || WM == 4, "a wave's rows of each matrix are one stored group");
            const int64_t first = m0 + mw * 32;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int64_t m = first + i * 16 + quarter * 4;
                float v[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float da;
                    activation(p.act, acc[i][t][r], v[r], da);
                    v[r] *= acc[i + WM / 2][t][r];
                }
                if (in) store4(y + m, (int)min((int64_t)4, p.M - m), v);
            }
            if (p.g8) {
                const int64_t saved_words = ((int64_t)p.M + 3) / 4, saved_groups = ((int64_t)p.M + SAMD_GATED_GROUP - 1) / SAMD_GATED_GROUP;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    uint32_t big = 0;
                    float v[2][4];
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            v[i][r] = first + i * 16 + quarter * 4 + r < p.M ? acc[b * (WM / 2) + i][t][r] : 0.0f;
                            big = max(big, __float_as_uint(v[i][r]) & 0x7fffffffu);
                        }
                    big = max(big, (uint32_t)__shfl_xor((int)big, 16, 64));
                    big = max(big, (uint32_t)__shfl_xor((int)big, 32, 64));
                    const GroupStep st = group_step(__uint_as_float(big), big, 127.0f, 1.0f / 127.0f);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int64_t m = first + i * 16 + quarter * 4;
                        uint32_t w = 0;
#pragma unroll
                        for (int r = 0; r < 4; ++r) w |= (st.bad ? 0u : (uint32_t)(int)rintf(v[i][r] * st.inv) & 255u) << (8 * r);
                        if (in && m < p.M) (b ? p.u8 : p.g8)[token * saved_words + m / 4] = w;
                    }
                    if (in && quarter == 0 && first < p.M) (b ? p.uscale : p.gscale)[token * saved_groups + first / SAMD_GATED_GROUP] = st.scale;
                }
            }
        }
    }
}

template <class X, bool BUF, int NW, int WT, int WM, int TW, int MW, int KS>
int launch_gemm_tile(const GroupProduct &p, int words, int groups, hipStream_t s) {
    constexpr int BT = 16 * WT * TW, OM = 16 * WM * MW / NW;
    const int64_t tblocks = ((int64_t)p.T + BT - 1) / BT, blocks = tblocks * (((int64_t)p.M + OM - 1) / OM);
    if (const int st = check_blocks(blocks, 64 * TW * MW * KS, "group product")) return st;
    auto go = [&](auto per) {
        hipLaunchKernelGGL((group_gemm_kernel<X, BUF, decltype(per)::value, NW, WT, WM, TW, MW, KS>), dim3((uint32_t)blocks),
                           dim3(64 * TW * MW * KS), 0, s, p, words, groups, (int)tblocks);
    };
    if (p.group == 32) go(std::integral_constant<int, 1>{});
    else if (p.group == 64) go(std::integral_constant<int, 2>{});
    else go(std::integral_constant<int, 4>{});
    return check_launch("group product");
}

}  // namespace samd
