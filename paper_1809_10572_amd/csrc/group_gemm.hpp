// Products of many tokens with 4-bit group-scaled weights on the matrix cores, and the gated block on two of them.
//
// A field minus its zero point is a whole number of -15..15, exact as a 16-bit float, so it is multiplied
// exactly and scaled once for each group and output, in 32-bit floats: no weight is ever rounded.  32-bit
// activations enter as three bf16 pieces (three instructions a product).
//
// A workgroup of TW x MW waves computes 16 WT TW tokens x 16 WM MW rows of W, a wave 16 WT x 16 WM.  Steps of 64
// values: x (copied) and the fields (decoded once for the workgroup) go through LDS, two buffers, the next
// step's loads in flight during this step's products.  A row of a buffer is 128 bytes, its 16-byte parts exchanged
// by (row / 2) % 8, so that the 16 rows which an operand's lanes read meet no bank twice.
// W is the first operand: a lane then ends with 4 consecutive rows of W for a token, which are stored together
// and are one word of the gated block's stored projections.
#pragma once

#include "group_device.hpp"

namespace samd {

constexpr int kGemmStep = 64;

// Index of 16-byte part `c` (0..7) of row `r` in a buffer.
__device__ __forceinline__ int part_at(int r, int c) { return r * 8 + (c ^ ((r >> 1) & 7)); }

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
        const uint32_t lo = w & 0x0f0f0f0fu, hi = (w >> 4) & 0x0f0f0f0fu;
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
template <class X, int ROWS, int THREADS>
struct TokenTile {
    static constexpr int kEach = ROWS * 8 / THREADS;   // 8-value parts of a thread
    Raw8<X> raw[kEach];

    __device__ __forceinline__ void load(const __amdgpu_buffer_rsrc_t &rx, const X *x, int64_t ld, int rows, int cols, int step,
                                         bool buffered) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int id = e * THREADS + threadIdx.x, k = step * kGemmStep + id % 8 * 8, row = min(id / 8, rows - 1);
            if (buffered) {
                const uint32_t at = k < cols ? ((uint32_t)row * (uint32_t)ld + k) * (uint32_t)sizeof(X) : 0xffffff00u;
#pragma unroll
                for (int c = 0; c < (int)sizeof(X) / 2; ++c)
                    raw[e].v[c] = __builtin_amdgcn_raw_buffer_load_b128(rx, at + 16 * c, 0, 0);
            } else {
                raw[e] = raw8(x + row * ld + k, cols - k);
            }
        }
    }

    template <int P>
    __device__ __forceinline__ void store(u32x4 (&to)[P][ROWS * 8], int cols, int step) {
        const bool ragged = step * kGemmStep + kGemmStep > cols;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int id = e * THREADS + threadIdx.x;
            if (ragged) clear_behind(raw[e], cols - (step * kGemmStep + id % 8 * 8));
            u32x4 piece[P];
            x_operand(raw[e], piece);
#pragma unroll
            for (int j = 0; j < P; ++j) to[j][part_at(id / 8, id % 8)] = piece[j];
        }
    }
};

// 4 neighbouring results of a row, `n` of them in range.
template <class X>
__device__ __forceinline__ void store4(X *p, int n, bool vec, const float (&v)[4]) {
    if (vec && n >= 4) {
        X t[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = (X)v[i];
        if constexpr (sizeof(X) == 4) *(u32x4 *)p = *(u32x4 *)t;
        else *(u32x2 *)p = *(u32x2 *)t;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = (X)v[i];
    }
}

// Every group of 4 columns of a row is on 4 elements.
inline bool rows4(const void *p, int type, int64_t ld) {
    const int64_t bytes = type == SAMD_F32 ? 16 : 8;
    return (uintptr_t)p % bytes == 0 && ld % 4 == 0;
}

template <class X, int PER, int NW, int WT, int WM, int TW, int MW>
__global__ __launch_bounds__(64 * TW * MW) void group_gemm_kernel(GroupProduct p, int words, int groups, int tblocks,
                                                                  bool buffered, bool vecy) {
    using H = std::conditional_t<std::is_same_v<X, half_t>, half_t, bf16_t>;
    constexpr int P = kPieces<X>, THREADS = 64 * TW * MW;
    constexpr int BT = 16 * WT * TW, BM = 16 * WM * MW;      // tokens and rows of W of a workgroup
    constexpr int OM = BM / NW;                               // rows of the result
    constexpr int WPT = BM * 8 / THREADS;                     // words of a thread and step
    constexpr int TPR = 8 / WPT;                              // threads of a row
    constexpr int SG = PER == 1 ? 2 : 1;                      // groups of a step
    static_assert(64 / TPR <= 16 * WM / NW || NW == 1, "a wave decodes rows of one matrix");
    __shared__ u32x4 xs[2][P][BT * 8], ws[2][BM * 8];
    __shared__ float ss[2][SG * BM];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
    const int wrow = threadIdx.x / TPR, part = threadIdx.x % TPR * WPT;
    const int a = __builtin_amdgcn_readfirstlane(matrix_of(wrow));
    const int row = result_row(wrow);
    const bool has_zero = p.w[0].zero != nullptr;
    const __amdgpu_buffer_rsrc_t rq = buffer_of(p.w[a].q + m0 * words, (int64_t)rows * words * 4);
    const __amdgpu_buffer_rsrc_t rz = buffer_of(p.w[a].zero + m0 * groups, has_zero ? (int64_t)rows * groups : 0);
    const uint32_t qrow = (uint32_t)row * (uint32_t)words, zrow = (uint32_t)row * (uint32_t)groups;
    // scales: thread i loads that of row i of the buffer
    static_assert(BM <= THREADS, "a thread loads the scales of one row");
    const int srow = result_row(threadIdx.x % BM);
    const bool scales = threadIdx.x < BM && srow < rows;
    const float *const sp = p.w[matrix_of(threadIdx.x % BM)].scale + (m0 + (scales ? srow : 0)) * groups;

    TokenTile<X, BT, THREADS> xt;
    uint32_t q[WPT];
    int z;
    float s[SG];
    auto load = [&](int step) {
        xt.load(rx, x, p.ldx, tokens, p.K, step, buffered);
        const uint32_t at = step < steps && row < rows ? (qrow + step * 8 + part) * 4 : 0xffffff00u;
        if constexpr (WPT == 4) {
            const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(rq, at, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = v[i];
        } else {
            const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(rq, at, 0, 0);
            q[0] = v[0], q[1] = v[1];
        }
        // a thread's words lie in one group
        const uint32_t g = (uint32_t)((step * kGemmStep + part * 8) / (32 * PER));
        z = has_zero ? (int)__builtin_amdgcn_raw_buffer_load_b8(rz, g < (uint32_t)groups ? zrow + g : 0xffffff00u, 0, 0) : 8;
#pragma unroll
        for (int c = 0; c < SG; ++c) {
            const int gs = step * kGemmStep / (32 * PER) + c;
            s[c] = scales && gs < groups ? sp[gs] : 0.0f;
        }
    };
    auto store = [&](int step, int buf) {
        xt.store(xs[buf], p.K, step);
#pragma unroll
        for (int i = 0; i < WPT; ++i)
            ws[buf][part_at(wrow, part + i)] = whole_values<H>(has_zero ? q[i] : q[i] ^ 0x88888888u, z);
        if (threadIdx.x < BM)
#pragma unroll
            for (int c = 0; c < SG; ++c) ss[buf][c * BM + threadIdx.x] = s[c];
    };

    f32x4 acc[WM][WT] = {}, sum[WM][WT] = {};
    auto flush = [&](int buf, int c) {
#pragma unroll
        for (int i = 0; i < WM; ++i) {
            const f32x4 f = *(const f32x4 *)&ss[buf][c * BM + (mw * WM + i) * 16 + quarter * 4];
#pragma unroll
            for (int t = 0; t < WT; ++t) {
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][t][r] = fmaf(f[r], sum[i][t][r], acc[i][t][r]);
                sum[i][t] = f32x4{};
            }
        }
    };
    auto multiply = [&](int buf, bool last_of_group) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            u32x4 av[WM];
#pragma unroll
            for (int i = 0; i < WM; ++i) av[i] = ws[buf][part_at((mw * WM + i) * 16 + low, c * 4 + quarter)];
#pragma unroll
            for (int t = 0; t < WT; ++t)
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const u32x4 bv = xs[buf][j][part_at((tw * WT + t) * 16 + low, c * 4 + quarter)];
#pragma unroll
                    for (int i = 0; i < WM; ++i) sum[i][t] = mfma<H>(av[i], bv, sum[i][t]);
                }
            if (PER == 1) {
                flush(buf, c);
                __builtin_amdgcn_sched_barrier(0);   // the halves overlapped would need more registers than there are
            }
        }
        if (PER > 1 && last_of_group) flush(buf, 0);
    };

    load(0);
    store(0, 0);
    __syncthreads();
    // two steps a turn: the buffers are known, and a group of 128 ends with the second (steps behind the last are zeros)
    for (int step = 0; step < steps; step += 2) {
        load(step + 1);
        multiply(0, PER == 2);
        store(step + 1, 1);
        __syncthreads();
        load(step + 2);
        multiply(1, true);
        store(step + 2, 0);
        __syncthreads();
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
                if (in) store4(y + m, (int)min((int64_t)4, p.M - m), vecy, v);
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
                if (in) store4(y + m, (int)min((int64_t)4, p.M - m), vecy, v);
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

template <class X, int NW, int WT, int WM, int TW, int MW>
int launch_gemm_tile(const GroupProduct &p, int words, int groups, hipStream_t s) {
    constexpr int BT = 16 * WT * TW, OM = 16 * WM * MW / NW;
    const int64_t tblocks = ((int64_t)p.T + BT - 1) / BT, blocks = tblocks * (((int64_t)p.M + OM - 1) / OM);
    if (blocks > INT32_MAX) {
        set_error("group product: T x M needs too many workgroups");
        return SAMD_EUNSUPPORTED;
    }
    const bool buffered = within_buffer(p.x, sizeof(X), std::min<int64_t>(p.T, BT), p.ldx, p.K);
    const bool vecy = rows4(p.y, p.type, p.ldy);
    auto go = [&](auto per) {
        hipLaunchKernelGGL((group_gemm_kernel<X, decltype(per)::value, NW, WT, WM, TW, MW>), dim3((uint32_t)blocks),
                           dim3(64 * TW * MW), 0, s, p, words, groups, (int)tblocks, buffered, vecy);
    };
    if (p.group == 32) go(std::integral_constant<int, 1>{});
    else if (p.group == 64) go(std::integral_constant<int, 2>{});
    else go(std::integral_constant<int, 4>{});
    return check_launch("group product");
}

}  // namespace samd
