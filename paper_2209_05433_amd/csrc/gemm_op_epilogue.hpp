// How a workgroup of four waves that owns 256 rows x 64 NB columns of a product leaves them through an operator (gfx950): each wave 128 x 32 NB,
// as NB x 4 blocks of 32 x 32.
#pragma once

#include "gemm_epilogue.hpp"
#include "gemm_op.hpp"

namespace fp8mm {
namespace {

// A lane holds 4 consecutive columns of a row per accumulator quad.  As in the plain epilogue the wave turns its rows around
// through its own piece of the idle LDS, here as the 32-bit sums: behind the turn a lane has 8 columns of a row, 8 (or 4) lanes a whole line of a
// 16-bit matrix, and everything else (factors, bias, the tensors that are read and kept, the activation) is done there, where every
// access to memory is 16 bytes a lane along the rows.  PAIR: the first half of the wave's columns are its outputs' gate, the other half
// the same outputs' second projection.  A lane's columns are the same in all rows: its bias and factors stay in registers, and so do
// its column sums, which meet the other lanes' of the wave's 128 rows at the end, in a fixed order.
//
// One wave a SIMD, nothing hides a load from memory.  What is read beside the product (z, g | u, the residual) therefore goes from
// memory straight into a ring in LDS, several steps ahead, a lane's 16 bytes where the same lane reads them; waits are counted by hand.  (As loads
// into registers the compiler waited for all of them at the first: its counts do not survive the branches around the stores.
// 8192 x 6144 gradients of a gated block with K = 2048: 343 us unasked, 267 in registers, 260 in the ring, 227 with no uncounted wait left; the
// product alone, to bf16, 170.)
constexpr int OP_RING = 69 * 1024, OP_RING_WAVE = 20 * 1024;            // LDS behind the turned rows: the waves' rings
constexpr int OP_ROW_FACTORS = 149 * 1024, OP_COLUMN_FACTORS = 153 * 1024, OP_AMAX = 157 * 1024;        // reciprocals of factors; a word per wave

// The vector-memory counter down to at most `allowed` (rounded down to a multiple of 4, 40 at most).
__device__ __forceinline__ void op_wait(int allowed)
{
    switch (allowed >> 2) {
        case 0: __builtin_amdgcn_s_waitcnt(0x0F70); break;      // vmcnt 0 (bits 3:0 and 15:14), the other counters free
        case 1: __builtin_amdgcn_s_waitcnt(0x0F74); break;
        case 2: __builtin_amdgcn_s_waitcnt(0x0F78); break;
        case 3: __builtin_amdgcn_s_waitcnt(0x0F7C); break;
        case 4: __builtin_amdgcn_s_waitcnt(0x4F70); break;
        case 5: __builtin_amdgcn_s_waitcnt(0x4F74); break;
        case 6: __builtin_amdgcn_s_waitcnt(0x4F78); break;
        case 7: __builtin_amdgcn_s_waitcnt(0x4F7C); break;
        case 8: __builtin_amdgcn_s_waitcnt(0x8F70); break;
        case 9: __builtin_amdgcn_s_waitcnt(0x8F74); break;
        default: __builtin_amdgcn_s_waitcnt(0x8F78); break;
    }
}

// 16 bytes a lane from base + off to 16 bytes a lane from lds_addr on.
__device__ __forceinline__ void op_direct_load(const void* p, unsigned lds_addr)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" :: "v"(p), "{m0}"(lds_addr) : "memory");
}

// SIDE: o.side is given (always, for the gradients), in 32 bits if F32.
template <int NB, int OP, bool SIDE, bool F32>
__device__ __forceinline__ void op_store_rows(v16f (&acc)[NB][4], uint8_t* smem, const OpArgs& o, void* D, int M, int N, int m0, int n0, int w)
{
    constexpr bool PAIR = OP == OP_GATED, BOTH = OP == OP_GATED_GRAD;
    constexpr int WN = 32 * NB, OUTW = PAIR ? WN / 2 : WN;      // columns of the wave, outputs of a row
    constexpr int ROWB = WN * 4 + 16;                           // padded LDS row
    constexpr int MBS = NB == 4 ? 1 : 2;                        // blocks of 32 rows that are turned at a time
    constexpr int LANES = OUTW / 8, ROWS = 64 / LANES;          // lanes that hold a row between them, rows at a time
    constexpr int G = BOTH ? 2 : 4;                             // rows that a lane finishes together: a step
    constexpr int STEPS = 32 * MBS / (ROWS * G), TURNS = 4 / MBS;
    constexpr int PARTS = (F32 ? 2 : 1), LOADS = G * (BOTH ? 2 : 1) * PARTS;    // requests of a step
    constexpr int AHEAD = OP_RING_WAVE / (LOADS * 1024);        // steps (5, or 2) that are requested ahead
    static_assert(64 % LANES == 0 && STEPS >= 1 && AHEAD >= 2 && OP_RING + 4 * OP_RING_WAVE <= OP_ROW_FACTORS, "whole rows; room for the ring");
    static_assert(4 * 32 * MBS * ROWB <= OP_RING, "room for the turned rows");
    const int l = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));      // (see store_tile)
    const int h = l >> 5, wn = w & 1;
    const int wave_m0 = m0 + (w >> 1) * 128, wave_n0 = n0 + wn * OUTW;
    const int col = wave_n0 + (l % LANES) * 8, left = N - col;
    uint8_t* blk = smem + w * (32 * MBS * ROWB);
    const int width = BOTH ? 2 * N : N;                         // of a row of o.side
    // no lane's columns reach over the edge (all, or none, of a lane's are outside), and rows of o.side begin on 16-byte boundaries
    const bool whole = N % 8 == 0 && ((uintptr_t)o.side & 15) == 0;

    // requests of step i of the wave's rows: the lane's 8 columns, or (outside) 8 inside a row, which nobody looks at
    const unsigned ring = (unsigned)(uintptr_t)LDS_PTR(void, smem) + OP_RING + w * OP_RING_WAVE;
    const int at_col = left >= 8 ? col : N - 8;
    auto request = [&](int i) __attribute__((always_inline)) {
        const unsigned slot = __builtin_amdgcn_readfirstlane(ring + (unsigned)(i % AHEAD) * (LOADS * 1024));
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int64_t at = (int64_t)min(wave_m0 + (i * G + g) * ROWS + l / LANES, M - 1) * width + at_col;
            const char* p = (const char*)o.side + at * (F32 ? 4 : 2);
#pragma unroll
            for (int k = 0; k < LOADS / G; ++k)
                op_direct_load(p + (k % PARTS) * 16 + (k / PARTS) * ((int64_t)N * (F32 ? 4 : 2)), slot + (g * (LOADS / G) + k) * 1024);
        }
    };
    if (SIDE && whole) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) request(i);
    }

    // Factors: one reciprocal for both operands where A has one factor; else those of the columns stay in LDS, beside the rows', in 64 bits
    // until their product is rounded.
    float fy[8], fu[8], bias[8];
    double* row_factors = (double*)(smem + OP_ROW_FACTORS) + w * 128;
    double* column_factors = (double*)(smem + OP_COLUMN_FACTORS) + w * 128 + (l % LANES) * (PAIR ? 16 : 8);
    {
        const double a_all = o.a_per_row ? 1.0 : 1.0 / (double)op_scalar(o.sA_dev);
        const bool one = o.b_factors == B_ONE;
        const double b_all = one ? 1.0 / (double)op_scalar(o.sB_dev) : 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = min(col + i, N - 1);
            const double y = one ? b_all : op_column_factor(o, N, c, false), u = !PAIR ? 0.0 : one ? b_all : op_column_factor(o, N, c, true);
            fy[i] = (float)(a_all * y);
            fu[i] = (float)(a_all * u);
            bias[i] = 0.0f;
            if (o.a_per_row) {
                *LDS_PTR(double, column_factors + i) = y;
                if (PAIR) *LDS_PTR(double, column_factors + 8 + i) = u;
            }
        }
        if (OP == OP_ACT && o.bias && left > 0) load_row<8>(o.bias, o.bias_dtype, col, left, bias);
    }
    if (o.a_per_row) {
#pragma unroll
        for (int i = 0; i < 2; ++i) *LDS_PTR(double, row_factors + 64 * i + l) = 1.0 / (double)o.sA_dev[min(wave_m0 + 64 * i + l, M - 1)];
    }
    const float sD = o.out_kind >= OUT_E4M3 && o.sD_dev ? op_scalar(o.sD_dev) : 1.0f;
    // What has been loaded so far is waited for here: at its first use, in the loop, the compiler would wait for all that is in flight, at every trip.
    if (OP == OP_ACT) {
#pragma unroll
        for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(bias[i]));
    }
    float column[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    unsigned top = 0;

    const bool inside = wave_m0 + 128 <= M && wave_n0 + OUTW <= N;
    // Sums of step i of the wave's rows (step `in_turn` of the turned ones) and what is beside them -> outputs.
    auto finish = [&](int in_turn, int i, const float (&a)[G * 8], const float (&b)[G * 8]) __attribute__((always_inline)) {
        float y[G * 8], u[G * 8];
        OutRows<G> t;
        t.col = col; t.left = left; t.rows = 0; t.whole = inside;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const uint8_t* src = blk + ((in_turn * G + g) * ROWS + l / LANES) * ROWB + (l % LANES) * 32;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const v4f s = *LDS_PTR(v4f, src + 16 * p);
                v4f s2 = {0.0f, 0.0f, 0.0f, 0.0f};
                if (PAIR) s2 = *LDS_PTR(v4f, src + OUTW * 4 + 16 * p);
#pragma unroll
                for (int e = 0; e < 4; ++e) { y[8 * g + 4 * p + e] = s[e]; u[8 * g + 4 * p + e] = s2[e]; }
            }
            const int row = wave_m0 + (i * G + g) * ROWS + l / LANES;
            t.row[g] = row;
            if (row < M && left > 0) t.rows |= 1u << g;
        }
        if (o.a_per_row) {
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const double f = *LDS_PTR(double, row_factors + (i * G + g) * ROWS + l / LANES);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    y[8 * g + e] *= (float)(f * *LDS_PTR(double, column_factors + e));
                    if (PAIR) u[8 * g + e] *= (float)(f * *LDS_PTR(double, column_factors + 8 + e));
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < G * 8; ++e) {
                y[e] *= fy[e % 8];
                if (PAIR) u[e] *= fu[e % 8];
            }
        }
        top = max(top, op_finish<G, 8, OP>(o, D, N, t, y, u, bias, a, b, sD));
        if (OP == OP_ACT_GRAD) {
#pragma unroll
            for (int e = 0; e < G * 8; ++e) column[e % 8] += y[e];
        }
    };
    // A wait for the requests of step i: those of the AHEAD - 1 steps behind it are younger, and the stores of as many steps, where all of them
    // happen (stores are counted like loads).  At the end the requests of the steps that are left.
    const int stores = G * ((OP == OP_ACT && o.kept ? (o.kept_dtype == FP8_F32 ? 2 : 1) : 0) + (BOTH ? 2 : 1) * (o.out_kind == OUT_F32 ? 2 : 1));
    const int younger = (AHEAD - 1) * (LOADS + (inside ? stores : 0));
    auto read_beside = [&](int i, float (&a)[G * 8], float (&b)[G * 8]) __attribute__((always_inline)) {
        const uint8_t* p = smem + OP_RING + w * OP_RING_WAVE + (i % AHEAD) * (LOADS * 1024) + l * 16;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int k = 0; k < LOADS / G; ++k) {
                const u32x4 v = *LDS_PTR(u32x4, p + (g * (LOADS / G) + k) * 1024);
                float* to = (k / PARTS ? b : a) + 8 * g;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (F32) to[4 * (k % PARTS) + e] = as_f32(v[e]);
                    else { to[2 * e] = as_f32(v[e] << 16); to[2 * e + 1] = as_f32(v[e] & 0xffff0000u); }
                }
            }
    };
    auto fence = [&]() __attribute__((always_inline)) { __atomic_signal_fence(__ATOMIC_SEQ_CST); };
#pragma unroll 1
    for (int turn = 0; turn < TURNS; ++turn) {
        auto turn_rows = [&](auto turn_tag) __attribute__((always_inline)) {
            constexpr int T = decltype(turn_tag)::value;
            if constexpr (T < TURNS) {
#pragma unroll
                for (int mb = 0; mb < MBS; ++mb)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const v16f& a = acc[nb][T * MBS + mb];
                            *LDS_PTR(v4f, blk + (mb * 32 + (l & 31)) * ROWB + (nb * 32 + 8 * q + 4 * h) * 4) = (v4f){a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]};
                        }
            }
        };
        switch (turn) {
            case 0: turn_rows(std::integral_constant<int, 0>{}); break;
            case 1: turn_rows(std::integral_constant<int, 1>{}); break;
            case 2: turn_rows(std::integral_constant<int, 2>{}); break;
            default: turn_rows(std::integral_constant<int, 3>{}); break;
        }
#pragma unroll 1
        for (int in_turn = 0; in_turn < STEPS; ++in_turn) {
            const int i = turn * STEPS + in_turn;
            float a[G * 8] = {}, b[G * 8] = {};
            if (SIDE && whole) {
                const int later = TURNS * STEPS - 1 - i;        // steps behind this one
                fence();
                op_wait(later < AHEAD - 1 ? later * LOADS : i < AHEAD ? (AHEAD - 1) * LOADS : younger);
                fence();
                read_beside(i, a, b);
                fence();
                __builtin_amdgcn_s_waitcnt(0xC07F);             // lgkmcnt(0): what was read is in registers, the slot is free
                if (later >= AHEAD) request(i + AHEAD);
                fence();
            } else if (SIDE && left > 0) {
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const int64_t row = min(wave_m0 + (i * G + g) * ROWS + l / LANES, M - 1);
                    float piece[8];
                    load_row<8>(o.side, o.side_dtype, row * width + col, left, piece);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        asm volatile("" : "+v"(piece[e]));      // (waited for on this path, not where the paths meet)
                        a[8 * g + e] = piece[e];
                    }
                    if (!BOTH) continue;
                    load_row<8>(o.side, o.side_dtype, row * width + N + col, left, piece);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        asm volatile("" : "+v"(piece[e]));
                        b[8 * g + e] = piece[e];
                    }
                }
            }
            finish(in_turn, i, a, b);
        }
    }
    if (OP == OP_ACT_GRAD && o.sums && wave_m0 < M) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int d = LANES; d <= 32; d <<= 1) column[e] += __shfl_xor(column[e], d, 64);
        if (l < LANES && left > 0) {
            float* out = o.sums + (size_t)(wave_m0 / 128) * N + col;
#pragma unroll
            for (int e = 0; e < 8; ++e) if (e < left) out[e] = column[e];
        }
    }
    if (o.amax_out) {
        // one atomic per workgroup, as in the plain epilogue
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, d, 64));
        unsigned* cells = (unsigned*)(smem + OP_AMAX);
        if (l == 0) *LDS_PTR(unsigned, cells + w) = top;
        __syncthreads();
        if (w == 0) op_commit_top(o, l < 4 ? *LDS_PTR(unsigned, cells + l) : 0u);
    }
}

// What the tile's end will read beside the product, brought into the caches while the matrix cores are busy: a word of every 128-byte line, so that
// the reads of all compute units at once at the end of a round do not wait for memory (3001 x 2048 x 6144 with a residual 73.8 -> 69.8 us).  Not for
// g | u, twice as much as the L2 holds for all tiles at work (8192 x 6144 gradients of a gated block: 273 -> 283 us).  `v` holds the words until touched() lets them go;
// nobody looks at them.  OP as below.
template <int NB, int OP>
struct OpTouch {
    static constexpr int MOST = NB * 2, OUT_N = 64 * NB;
    unsigned v[MOST];
    __device__ __forceinline__ void touch(const OpArgs& o, int M, int N, int m0, int n0, int tid)
    {
        if (!o.side || o.op == OP_GATED_GRAD) return;
        const int esz = o.side_dtype == FP8_F32 ? 4 : 2, lines = OUT_N * esz / 128;
#pragma unroll
        for (int j = 0; j < MOST; ++j) {
            if (j >= lines) continue;
            const int line = j * 256 + tid;
            const int64_t at = (int64_t)min(m0 + line / lines, M - 1) * N + min(n0 + line % lines * (128 / esz), N - 1);
            v[j] = *(const unsigned short*)((const char*)o.side + at * esz);
        }
    }
    __device__ __forceinline__ void touched()
    {
#pragma unroll
        for (int j = 0; j < MOST; ++j) asm volatile("" :: "v"(v[j]));
    }
};
template <int NB> struct OpTouch<NB, 0> { };
template <int NB> struct OpTouch<NB, 2> { };

// OP of the tile: 1 the product alone, 2 the gated block, 3 the gradients.
template <int NB, int OP>
__device__ __forceinline__ void op_store_tile(v16f (&acc)[NB][4], uint8_t* smem, const OpArgs& o, void* D, int M, int N, int m0, int n0, int w)
{
    const bool f32 = o.side_dtype == FP8_F32;
    if constexpr (OP == 1) {
        if (!o.side) op_store_rows<NB, OP_ACT, false, false>(acc, smem, o, D, M, N, m0, n0, w);
        else if (f32) op_store_rows<NB, OP_ACT, true, true>(acc, smem, o, D, M, N, m0, n0, w);
        else op_store_rows<NB, OP_ACT, true, false>(acc, smem, o, D, M, N, m0, n0, w);
    } else if constexpr (OP == 2) {
        op_store_rows<NB, OP_GATED, false, false>(acc, smem, o, D, M, N, m0, n0, w);
    } else if (o.op == OP_ACT_GRAD) {
        if (f32) op_store_rows<NB, OP_ACT_GRAD, true, true>(acc, smem, o, D, M, N, m0, n0, w);
        else op_store_rows<NB, OP_ACT_GRAD, true, false>(acc, smem, o, D, M, N, m0, n0, w);
    } else {
        if (f32) op_store_rows<NB, OP_GATED_GRAD, true, true>(acc, smem, o, D, M, N, m0, n0, w);
        else op_store_rows<NB, OP_GATED_GRAD, true, false>(acc, smem, o, D, M, N, m0, n0, w);
    }
}

}  // namespace
}  // namespace fp8mm
