// The input gradient of products with 4-bit group-scaled weights on the matrix cores: dx = dy W (+ dy2 W2).
//
// The sum runs over the rows of W, and a group's scale differs from row to row, so it is part of the summed product
// and has to be multiplied into an operand in 32-bit floats, one of two ways:
//   into the weights   s (u - z), rounded once to 32 bits, then: for bf16 rounded to one bf16 (off by at most 2^-8 of each
//                      weight, as the types of dy and dx are); for f16 two bf16 (cut off at 8 bits, the rest rounded), dy as
//                      two that hold its 11 bits, three instructions a product, the lower parts' left out (in all at most
//                      9/8 2^-14 of each product, where the result's own rounding is 2^-11); for f32 three, as is dy, the
//                      six largest of their products (the others at most 2^-21 of each, about 2^-24 as a rule)
//   into dy            s dy for each group of the tile's columns, as two bf16 (f16, 16 bits and more) or three (f32, all 24);
//                      u - z is a whole number, exact as one bf16: two or three instructions, but dy is converted
//                      once for each group, 64 columns at most.  Groups of 64 and 128, and few tokens in f32: 512 x
//                      4096 x 4096 f32 113 us to 91; with groups of 32 2048 tokens take 687 us so and 467 the other way
// (a bf16 holds any float's range; an f16 operand would lose small scales).  Everything is summed in 32-bit floats, both
// pairs into one sum, and rounded once.
//
// A workgroup computes 16 WT TW tokens x 16 WM MW columns of W with TW x MW waves for each of KS slices of the sum, steps
// of 64 rows of W through LDS as in the products of many tokens.  The matrix instruction wants neighbouring rows of W side
// by side, the words hold neighbouring columns: the words go into LDS as they are (read straight into the threads that
// decode them, each row of each word and its scale was a load: 168 us against 110 for 2048 x 4096 x 4096 bf16, one tile), and a
// thread then takes the same KPT columns of eight rows and writes KPT operand parts of eight rows each, so that
// the transposition costs nothing but its choice of pairs.
//
// Measured (graph of calls, 4096 x 4096 weights, signed groups of 128): 2048 tokens bf16 92 us (745 TFLOP/s of the
// 1150 that a large library product reaches), f32 355 us, 1024 tokens f16 105 us; 128 tokens bf16 28 us, f16 33, f32 36.
// Bound by what lies between two barriers of a step (operands out of LDS, the next step's decoding and writes), only in
// part under the other waves' products.  Few tokens are bound by the chain of steps of a workgroup, whose number only
// the slices cut: as many as LDS holds.
#include <hip/hip_runtime.h>

#include "group_gemm.hpp"

namespace samd {

namespace {

// bf16 pieces of dy, or of dy times a scale.
template <class X>
constexpr int kGradPieces = sizeof(X) == 4 ? 3 : std::is_same_v<X, half_t> ? 2 : 1;

// The upper halves of two floats: bf16 by cutting off.
__device__ __forceinline__ uint32_t upper_halves(float a, float b) {
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}

__device__ __forceinline__ float behind_upper_half(float v) { return v - __uint_as_float(__float_as_uint(v) & 0xffff0000u); }

// 8 floats as P bf16 operands: all but the last by cutting, the last rounded.
template <int P>
__device__ __forceinline__ void pieces_of(float (&v)[8], u32x4 (&out)[P]) {
#pragma unroll
    for (int j = 0; j < P; ++j) {
        if (j == P - 1) {
            Eight<bf16_t> h;
#pragma unroll
            for (int i = 0; i < 8; ++i) h.v[i] = (bf16_t)v[i];
            out[j] = __builtin_bit_cast(u32x4, h);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) out[j][i] = upper_halves(v[2 * i], v[2 * i + 1]);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = behind_upper_half(v[i]);
        }
    }
}

// 8 values of dy, or of dy times their rows' scales, as operands.
template <class X, int P, class F>
__device__ __forceinline__ void grad_operand(const Raw8<X> &raw, u32x4 (&out)[P], F &&scale) {
    const Eight<X> x = __builtin_bit_cast(Eight<X>, raw);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)x.v[i] * scale(i);
    pieces_of(v, out);
}

// GX: groups of a tile whose scales go into dy; 0: the scales go into the weights.
template <class X, bool SIGNED, bool BUF, int GX, int WT, int WM, int TW, int MW, int KS>
__global__ __launch_bounds__(64 * TW * MW * KS) void group_grad_kernel(GroupGrad p, int words, int groups, int gshift,
                                                                       int tblocks) {
    constexpr int P = kGradPieces<X>, THREADS = 64 * TW * MW;
    constexpr int BT = 16 * WT * TW, BN = 16 * WM * MW;
    constexpr int DECODERS = THREADS < BN * 4 ? THREADS : BN * 4;   // threads that decode
    constexpr int KPT = BN * 8 / DECODERS;   // columns of a thread: a half or a quarter of a word
    static_assert(KPT == 2 || KPT == 4, "columns of a thread");
    constexpr int DY = GX ? GX : 1;          // operands of dy
    static_assert(MW % DY == 0, "a wave's columns lie in one group of the tile");
    constexpr int PW = GX ? 1 : P;           // operands of W
    constexpr int WORDS = BN / 8, GROUPS = BN / 32;   // of a row of the tile; the most groups
    constexpr bool kByScale = SIGNED && GX == 0;      // s u - 8 s, where 8 s is exact
    constexpr int kScaleRow = kGemmStep + 8;          // of one group's column, a quarter of the banks further each
    struct Buffers {
        u32x4 x[2][DY][P][BT * 8], w[2][PW][BN * 8];
        u32x4 q[2][kGemmStep * WORDS / 4];        // words as they are stored, 64 rows
        f32x2 s[2][GROUPS * kScaleRow];           // scales, and -(1024 + z) and -(64 + z) as two f16, or -8 s
    };
    static_assert((KS - 1) * BT * BN * 4 <= (int)sizeof(Buffers) * KS, "the slices' sums meet in the buffers");
    __shared__ Buffers all[KS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % (TW * MW);
    const int slice = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / (TW * MW), tid = threadIdx.x - slice * THREADS;
    auto &xs = all[slice].x;
    auto &ws = all[slice].w;
    const int quarter = lane >> 4, low = lane & 15, tw = wave % TW, mw = wave / TW;
    const uint32_t tile = tile_of(blockIdx.x, gridDim.x);
    const int64_t t0 = (int64_t)(tile % tblocks) * BT, k0 = (int64_t)(tile / tblocks) * BN;
    const int tokens = (int)min((int64_t)BT, p.T - t0);
    const int single = (p.M + kGemmStep - 1) / kGemmStep, steps = p.dy[1] ? 2 * single : single;   // of both pairs

    // Position n of a slice is a step of both pairs' rows; those behind the last are zeros.
    auto step_of = [&](int n) { return __builtin_amdgcn_readfirstlane(2 * slice + n / 2 * 2 * KS + n % 2); };

    // On the way in, a thread takes four neighbouring words of a row and the scale of a row and group.
    constexpr int UNITS = kGemmStep * WORDS / 4;
    const int urow = tid % UNITS / (WORDS / 4), ucol = tid % (WORDS / 4);
    const int tile_groups = max(1, BN >> gshift), g0 = (int)(k0 >> gshift);
    const int srow = tid % kGemmStep, sgroup = min(tid / kGemmStep, tile_groups - 1);
    struct Words {
        u32x4 q;
        float s;
        uint32_t z;
    } fw;
    auto load_words = [&](int n) SAMD_INLINE {
        int step = step_of(n);
        asm("" : "+s"(step));   // addresses from one scalar each turn, not a register carried for each of them
        const bool second = step >= single && p.dy[1];
        // the step's rows of W; rows behind the last read as zeros (of scale 0)
        const int64_t m0 = min((int64_t)(second ? step - single : step) * kGemmStep, (int64_t)p.M);
        const int64_t rows = min((int64_t)kGemmStep, p.M - m0);
        const GroupW &w = p.w[second ? 1 : 0];
        const __amdgpu_buffer_rsrc_t rq = buffer_of(w.q + m0 * words, rows * words * 4);
        const __amdgpu_buffer_rsrc_t rs = buffer_of(w.scale + m0 * groups, rows * groups * 4);
        const __amdgpu_buffer_rsrc_t rz = byte_buffer_of(w.zero + m0 * groups, SIGNED ? 0 : rows * groups);
        fw.q = __builtin_amdgcn_raw_buffer_load_b128(rq, ((uint32_t)urow * (uint32_t)words + (uint32_t)(k0 / 8) + ucol * 4) * 4, 0, 0);
        const uint32_t g = (uint32_t)srow * (uint32_t)groups + (uint32_t)min(g0 + sgroup, groups - 1);
        fw.s = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, g * 4, 0, 0));
        if (!SIGNED) fw.z = __builtin_amdgcn_raw_buffer_load_b8(rz, g, 0, 0);
    };
    // Four words of row 8 c + j: the reads of one j take all c and two neighbouring fours, which fill the 256 bytes of
    // all banks; the writes take 16 of one c, for which the places are exchanged by the rest.
    auto four_at = [&](int c, int j, int four) SAMD_INLINE {
        const int rest = j * (WORDS / 8) + four / 2;
        return rest * 16 + ((c * 2 + four % 2) ^ (rest % 8 * 2));
    };
    auto scale_at = [&](int c, int j, int group) SAMD_INLINE { return group * kScaleRow + j * 8 + c; };
    auto store_words = [&](int buf) SAMD_INLINE {
        all[slice].q[buf][four_at(urow / 8, urow % 8, ucol)] = fw.q;
        all[slice].s[buf][scale_at(srow / 8, srow % 8, sgroup)] = f32x2{fw.s, kByScale ? -8.0f * fw.s : zero_point_word<SIGNED>(fw.z)};
    };
    // On to the operands, a thread takes KPT columns of 8 rows; eight neighbouring threads different rows.
    const int chunk = tid % 8, column = (tid / 8 % WORDS) * 8 + tid % DECODERS / BN * KPT;
    const int word = column / 8, shift = column % 8 * 4, sgroup_of = column >> gshift;
    // four fields: the bytes that hold them into the lower bytes of two halves
    const uint32_t spread = shift ? 0x0c030c02u : 0x0c010c00u;
    auto decode = [&](int buf) SAMD_INLINE {
        if (DECODERS < THREADS && tid >= DECODERS) return;
        const uint32_t one = as_is(SIGNED ? 0x64086408u : 0x64006400u), sixteen = SIGNED ? as_is(0x64806480u) : one;
        const float unit = as_float(1.0f);
        float v[KPT][8];
        const uint32_t *q = (const uint32_t *)all[slice].q[buf];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t w = q[four_at(chunk, j, word / 4) * 4 + word % 4];
            const f32x2 s = all[slice].s[buf][scale_at(chunk, j, sgroup_of)];
            if constexpr (kByScale) {   // (f16, groups of 32, 128 tokens: 50 us, the other way 54)
                const uint32_t u = ((w ^ 0x88888888u) >> shift) & (KPT == 4 ? 0xffffu : 0xffu);
                const uint32_t lo = as_is(u & 0x0f0f0f0fu), hi = as_is((u >> 4) & 0x0f0f0f0fu);
#pragma unroll
                for (int c = 0; c < KPT; c += 2) {
                    v[c][j] = fmaf(s[0], (float)((lo >> (4 * c)) & 255u), s[1]);
                    v[c + 1][j] = fmaf(s[0], (float)((hi >> (4 * c)) & 255u), s[1]);
                }
            } else {   // u - z exactly, by a multiply-add on the f16 1024 + u or 1024 + 16 u; then times its scale: s z is not exact
                const half2_t less = __builtin_bit_cast(half2_t, __float_as_uint(s[1]));
                const uint32_t u = KPT == 4 ? __builtin_amdgcn_perm(0u, w, spread) : w >> shift;
                const half2_t even = __builtin_bit_cast(half2_t, (u & 0x000f000fu) ^ one);
                const half2_t odd = __builtin_bit_cast(half2_t, (u & 0x00f000f0u) ^ sixteen);
#pragma unroll
                for (int c = 0; c < KPT; c += 2) {
                    v[c][j] = (GX ? 1.0f : s[0]) * fmaf((float)even[c / 2], unit, (float)less[0]);
                    v[c + 1][j] = (GX ? 1.0f : s[0]) * fmaf((float)odd[c / 2], 0.0625f, (float)less[1]);
                }
            }
        }
#pragma unroll
        for (int c = 0; c < KPT; ++c) {
            u32x4 piece[PW];
            if constexpr (GX != 0) {   // whole numbers of at most 4 bits
#pragma unroll
                for (int i = 0; i < 4; ++i) piece[0][i] = upper_halves(v[c][2 * i], v[c][2 * i + 1]);
            } else {
                pieces_of(v[c], piece);
            }
#pragma unroll
            for (int j = 0; j < PW; ++j) ws[buf][j][part_at(column + c, chunk)] = piece[j];
        }
    };
    TokenTile<X, BT, THREADS, BUF> fx;
    auto load_x = [&](int n) SAMD_INLINE {
        int step = step_of(n);
        asm("" : "+s"(step));
        const bool second = step >= single && p.dy[1];
        const X *x = (const X *)(second ? p.dy[1] : p.dy[0]) + t0 * p.lddy;
        const __amdgpu_buffer_rsrc_t rx = buffer_of(x, ((int64_t)(tokens - 1) * p.lddy + p.M) * (int64_t)sizeof(X));
        fx.load(rx, x, p.lddy, tokens, p.M, second ? step - single : step, tid);
    };
    auto store_x = [&](auto ragged, int n, int buf) SAMD_INLINE {
        const int step = step_of(n);
        const int at_step = p.dy[1] && step >= single ? step - single : step;
        if constexpr (GX != 0) {   // a thread's values are those of eight rows of W
#pragma unroll
            for (int g = 0; g < DY; ++g) {
                float scale[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) scale[j] = all[slice].s[buf][scale_at(chunk, j, g)][0];
                fx.template store<decltype(ragged)::value>(xs[buf][g], p.M, at_step, tid, [&](const Raw8<X> &r, u32x4(&o)[P]) SAMD_INLINE {
                    grad_operand(r, o, [&](int j) SAMD_INLINE { return scale[j]; });
                });
            }
        } else {
            fx.template store<decltype(ragged)::value>(xs[buf][0], p.M, at_step, tid, [](const Raw8<X> &r, u32x4(&o)[P]) {
                if constexpr (std::is_same_v<X, half_t>) grad_operand(r, o, [](int) { return 1.0f; });
                else x_operand(r, o);
            });
        }
    };

    const int at[2] = {part_at(low, quarter), part_at(low, 4 + quarter)};   // the same in every 16 rows
    f32x4 acc[WM][WT] = {};
    u32x4 av[2][PW][WM];
    auto operands = [&](int buf) SAMD_INLINE {
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int j = 0; j < PW; ++j)
#pragma unroll
                for (int i = 0; i < WM; ++i) av[c][j][i] = ws[buf][j][(mw * WM + i) * 128 + at[c]];
    };
    auto multiply = [&](auto &&x_of, int from, int to) SAMD_INLINE {
#pragma unroll
        for (int t = from; t < to; ++t)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const u32x4 bv = x_of(c, j, t);
#pragma unroll
                    for (int h = 0; h < (GX ? 1 : P - j); ++h)   // pieces j and h: 2^-8(j + h) of the product
#pragma unroll
                        for (int i = 0; i < WM; ++i) acc[i][t] = mfma<bf16_t>(av[c][h][i], bv, acc[i][t]);
                }
    };

    // Position n's operands are made while those of n - 1 are multiplied, its words come into LDS one position
    // earlier.  Turns of two positions, so that the buffers are known; all slices take as many.
    const int turns = (steps + 2 * KS - 1) / (2 * KS);
    load_words(0);
    load_x(0);
    store_words(0);
    load_words(1);
    __syncthreads();
    store_x(std::true_type{}, 0, 0);
    load_x(1);
    decode(0);
    store_words(1);
    load_words(2);
    __syncthreads();
    auto ahead = [&](auto ragged, int n, int buf) SAMD_INLINE {   // while position n, in buffer buf, is multiplied
        store_x(ragged, n + 1, buf ^ 1);
        decode(buf ^ 1);
        store_words(buf);
        load_x(n + 2);
        load_words(n + 3);
    };
    auto both = [&](auto ragged, int n, int buf) SAMD_INLINE {
        auto x_of = [&](int c, int j, int t) SAMD_INLINE { return xs[buf][mw * DY / MW][j][(tw * WT + t) * 128 + at[c]]; };
        operands(buf);
        multiply(x_of, 0, WT / 2);
        ahead(ragged, n, buf);
        multiply(x_of, WT / 2, WT);
        __syncthreads();
    };
    auto turn_of = [&](auto ragged, int n) SAMD_INLINE {
        both(ragged, n, 0);
        both(ragged, n + 1, 1);
    };
    int turn = 0;
    const bool whole = p.M % kGemmStep == 0;   // else each pair ends with a ragged step
    for (; turn < turns && whole && step_of(2 * turn + 2) < steps; ++turn) turn_of(std::false_type{}, 2 * turn);
    for (; turn < turns; ++turn) turn_of(std::true_type{}, 2 * turn);
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
#pragma unroll
        for (int i = 0; i < WM; ++i) {
            const int64_t k = k0 + (mw * WM + i) * 16 + quarter * 4;
            const float v[4] = {acc[i][t][0], acc[i][t][1], acc[i][t][2], acc[i][t][3]};
            if (token < p.T) store4((X *)p.dx + token * p.lddx + k, (int)min((int64_t)4, p.K - k), v);
        }
    }
}

template <class X, bool BUF, int GX, int WT, int WM, int TW, int MW, int KS>
int launch_grad_tile(const GroupGrad &p, hipStream_t s) {
    constexpr int BT = 16 * WT * TW, BN = 16 * WM * MW;
    const int words = (int)row_words(p.K, 4), groups = (p.K + p.group - 1) / p.group;
    const int gshift = p.group == 32 ? 5 : p.group == 64 ? 6 : 7;
    const int64_t tblocks = ((int64_t)p.T + BT - 1) / BT, blocks = tblocks * (((int64_t)p.K + BN - 1) / BN);
    if (const int st = check_blocks(blocks, 64 * TW * MW * KS, "samd_group_matmul_grad")) return st;
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(64 * TW * MW * KS), 0, s, p, words, groups, gshift, (int)tblocks);
    };
    p.w[0].zero ? go(group_grad_kernel<X, false, BUF, GX, WT, WM, TW, MW, KS>)
                : go(group_grad_kernel<X, true, BUF, GX, WT, WM, TW, MW, KS>);
    return check_launch("samd_group_matmul_grad");
}

// A workgroup fills a CU, so a tile costs its time for each round of 256 workgroups; the units are about the microseconds
// measured for M = 4096 (they grow with M alike).  Rows of dy at odd addresses, an odd M of a 16-bit type, have the smallest
// tile alone: 2048 x 4095 x 4096 bf16 takes 309 us where 4096 takes 92, 1024 tokens f16 208 and 105.
template <class X>
int launch_grad_of(const GroupGrad &p, hipStream_t s) {
    const int64_t rows = std::min<int64_t>(p.T, 256);
    const bool buffered = within_buffer(p.dy[0], sizeof(X), rows, p.lddy, p.M) &&
                          (!p.dy[1] || within_buffer(p.dy[1], sizeof(X), rows, p.lddy, p.M));
    auto cost = [&](int64_t tokens, int64_t columns, int64_t unit) {
        const int64_t blocks = ((p.T + tokens - 1) / tokens) * ((p.K + columns - 1) / columns);
        return (blocks + 255) / 256 * unit;
    };
    if constexpr (std::is_same_v<X, bf16_t>) {
        if (!buffered) return launch_grad_tile<X, false, 0, 2, 4, 2, 1, 4>(p, s);
        const int64_t small = cost(64, 64, 29), middle = cost(128, 128, 55), large = cost(256, 128, 91);
        if (large < middle && large < small) return launch_grad_tile<X, true, 0, 4, 4, 4, 2, 1>(p, s);
        if (middle < small) return launch_grad_tile<X, true, 0, 4, 4, 2, 2, 2>(p, s);
        return launch_grad_tile<X, true, 0, 2, 4, 2, 1, 4>(p, s);
    } else if constexpr (std::is_same_v<X, half_t>) {
        if (p.group == 32) {
            if (!buffered) return launch_grad_tile<X, false, 0, 2, 2, 2, 2, 2>(p, s);
            if (cost(128, 128, 116) < cost(64, 64, 54)) return launch_grad_tile<X, true, 0, 2, 4, 4, 2, 1>(p, s);
            return launch_grad_tile<X, true, 0, 2, 2, 2, 2, 2>(p, s);
        }
        if (!buffered) return launch_grad_tile<X, false, 1, 2, 2, 2, 2, 2>(p, s);
        const int64_t small = cost(32, 64, 37), middle = cost(64, 64, 49), large = cost(256, 64, 108);
        if (large < middle && large < small) return launch_grad_tile<X, true, 1, 4, 2, 4, 2, 1>(p, s);
        if (middle < small) return launch_grad_tile<X, true, 1, 2, 2, 2, 2, 2>(p, s);
        return launch_grad_tile<X, true, 1, 1, 2, 2, 2, 4>(p, s);
    } else {
        if (p.group == 32) {
            const int64_t small = cost(32, 64, 52), middle = cost(64, 64, 85), large = cost(64, 128, 114);
            if (!buffered) return launch_grad_tile<X, false, 2, 1, 2, 2, 2, 2>(p, s);
            if (large < middle && large < small) return launch_grad_tile<X, true, 0, 2, 2, 2, 4, 1>(p, s);
            if (middle < small) return launch_grad_tile<X, true, 2, 1, 2, 4, 2, 1>(p, s);
            return launch_grad_tile<X, true, 2, 1, 2, 2, 2, 2>(p, s);
        }
        const int64_t small = cost(32, 64, 40), middle = cost(64, 64, 56), large = cost(128, 64, 89);
        if (!buffered) return launch_grad_tile<X, false, 1, 1, 2, 2, 2, 2>(p, s);
        if (large < middle && large < small) return launch_grad_tile<X, true, 1, 2, 2, 4, 2, 1>(p, s);
        if (middle < small) return launch_grad_tile<X, true, 1, 2, 2, 2, 2, 2>(p, s);
        return launch_grad_tile<X, true, 1, 1, 2, 2, 2, 3>(p, s);
    }
}

}  // namespace

int launch_group_matmul_grad(const GroupGrad &p, hipStream_t s) {
    if (p.type == SAMD_F32) return launch_grad_of<float>(p, s);
    if (p.type == SAMD_F16) return launch_grad_of<half_t>(p, s);
    return launch_grad_of<bf16_t>(p, s);
}

}  // namespace samd
