// How a workgroup of four waves that owns 256 rows x 64 NB columns of the logits leaves them (gemm_loss.hpp; gfx950): each wave 128 x 32 NB, as NB x 4 blocks of
// 32 x 32.
#pragma once

#include "gemm_loss.hpp"
#include "gemm_op_epilogue.hpp"

namespace fp8mm {
namespace {

// What the tile's end needs of its 256 rows: a thread asks for one row's while the last stage is multiplied, in four registers, and leaves it in LDS when the
// slabs are done with.  (A lane's own four rows, in sixteen registers, spilled 92 bytes of every thread: the gradient of 4096 x 50257 x 2048 762 us instead of 737.)
template <int OP>
struct LossRows {
    int64_t label;
    float lse, dloss;
    __device__ __forceinline__ void fetch(const LossArgs& o, int M, int m0, int w)
    {
        const int row = min(m0 + w * 64 + (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)), M - 1);
        label = o.labels[row];
        if (OP == 5) { lse = o.lse[row]; dloss = o.dloss[o.dloss_per_row ? row : 0]; }
    }
    // (behind a barrier; ends with one)
    __device__ __forceinline__ void leave(const LossArgs& o, int N, uint8_t* smem, int w) const
    {
        const int row = w * 64 + (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
        const int64_t c = column_of_label(o, label);
        const int column = c < N ? (int)c : -2;
        if (OP == 4) {
            *LDS_PTR(int, smem + OP_ROW_FACTORS + row * 4) = column;
        } else {
            const LossRow r = loss_row(o, lse, dloss, label);
            *LDS_PTR(v4f, smem + OP_ROW_FACTORS + row * 16) = (v4f){r.lse2, r.scale, r.dloss, as_f32((unsigned)column)};
        }
        __syncthreads();
    }
};
template <int NB> struct OpTouch<NB, 4> : LossRows<4> { };
template <int NB> struct OpTouch<NB, 5> : LossRows<5> { };

// The sums of the wave's rows 32 mb .. 32 mb + 31.  (The ends below walk the four blocks of rows in a loop: unrolled, a tile's end was four times the code, which
// every tile fetches anew.)
template <int NB>
__device__ __forceinline__ void sums_of(const v16f (&acc)[NB][4], int mb, float (&x)[NB * 16])
{
    // (the empty statement, another one at the end of each branch, keeps the branches apart: joined they would read the sums by an index, from memory)
    auto take = [&](auto tag) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NB * 16; ++i) x[i] = acc[i >> 4][decltype(tag)::value][i & 15];
        asm volatile("; rows %1" : "+v"(x[0]) : "n"(32 * decltype(tag)::value));
    };
    switch (mb) {
        case 0: take(std::integral_constant<int, 0>{}); break;
        case 1: take(std::integral_constant<int, 1>{}); break;
        case 2: take(std::integral_constant<int, 2>{}); break;
        default: take(std::integral_constant<int, 3>{}); break;
    }
}
// The column of a lane's value i of its row, of lanes h = 0 .. 31 and 32 .. 63.
__device__ __forceinline__ int loss_column(int i, int h) { return (i >> 4) * 32 + ((i >> 2) & 3) * 8 + 4 * h + (i & 3); }

// The loss: straight from the registers.  A lane holds half of a row's columns in each of its four rows (lane l and l + 32 the two halves), so a
// row's pair over the wave's columns takes one exchange between lanes, and no logit goes through LDS.
// PLAIN: one positive factor for all, no columns outside.
template <int NB, bool PLAIN>
__device__ __forceinline__ void loss_store_pairs(v16f (&acc)[NB][4], uint8_t* smem, const LossArgs& o, double a_all, double b_all, int M, int N, int wave_m0,
                                                 int wave_n0, int w, int l)
{
    const int h = l >> 5;
    double* columns = (double*)(smem + OP_COLUMN_FACTORS) + w * 128;
    if (!PLAIN && o.b_factors != B_ONE) {
#pragma unroll
        for (int i = 0; i < (NB + 1) / 2; ++i)
            if (64 * i + l < 32 * NB) *LDS_PTR(double, columns + 64 * i + l) = 1.0 / (double)o.sB_dev[min(wave_n0 + 64 * i + l, N - 1)];
    }
    // narrow tiles behind wide ones (both widths in one launch) have two blocks of columns where a wide one has one
    const int64_t block = NB == 4 ? wave_n0 / 128 : wave_n0 / 64 - 2 * o.wide_cols;
    LossPair* pairs = (LossPair*)o.partials + block * M;
    float* targets = loss_targets(o, M, N);
    const float f = (float)(a_all * b_all), f2 = (float)(a_all * b_all * (double)kLog2e);
#pragma unroll 1
    for (int mb = 0; mb < 4; ++mb) {
        const int row = wave_m0 + 32 * mb + (l & 31);
        const int column = *LDS_PTR(int, smem + OP_ROW_FACTORS + ((w >> 1) * 128 + 32 * mb + (l & 31)) * 4);
        const int label = column >= wave_n0 && column < wave_n0 + 32 * NB ? column - wave_n0 : -1;
        float t[NB * 16];
        sums_of<NB>(acc, mb, t);
        if (!PLAIN) {
            const double fa = o.a_per_row ? 1.0 / (double)o.sA_dev[min(row, M - 1)] : a_all;
#pragma unroll
            for (int i = 0; i < NB * 16; ++i) t[i] *= (float)(fa * (o.b_factors == B_ONE ? b_all : *LDS_PTR(double, columns + loss_column(i, h))));
        }
        // the label's column is in few of the tiles: its logit, by the same factor
        if (__any(label >= 0)) {
            float z = 0.0f;
#pragma unroll
            for (int i = 0; i < NB * 16; ++i) z = label == loss_column(i, h) ? t[i] : z;
            if (label >= 0 && ((label >> 2) & 1) == h && row < M) targets[row] = PLAIN ? z * f : z;
        }
        if (!PLAIN) {
#pragma unroll
            for (int i = 0; i < NB * 16; ++i) t[i] = wave_n0 + loss_column(i, h) < N ? t[i] : -__builtin_inff();
        }
        const LossPair p = loss_pair<NB * 16, 2, 32>(t, PLAIN ? f2 : kLog2e);
        if (l < 32 && row < M) pairs[row] = p;
    }
}

template <int NB>
__device__ __forceinline__ void loss_store_pairs(v16f (&acc)[NB][4], uint8_t* smem, const LossArgs& o, int M, int N, int m0, int n0, int w)
{
    const int l = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));      // (see store_tile)
    const int wave_m0 = m0 + (w >> 1) * 128, wave_n0 = n0 + (w & 1) * (32 * NB);
    if (wave_n0 >= N) return;
    const double a_all = o.a_per_row ? 1.0 : 1.0 / (double)op_scalar(o.sA_dev), b_all = o.b_factors == B_ONE ? 1.0 / (double)op_scalar(o.sB_dev) : 1.0;
    // (the largest logit belongs to the largest sum where the factor is positive)
    if (wave_n0 + 32 * NB <= N && !o.a_per_row && o.b_factors == B_ONE && a_all * b_all > 0.0) loss_store_pairs<NB, true>(acc, smem, o, a_all, b_all, M, N, wave_m0, wave_n0, w, l);
    else loss_store_pairs<NB, false>(acc, smem, o, a_all, b_all, M, N, wave_m0, wave_n0, w, l);
}

// The gradient: as the plain epilogue leaves outputs, everything in the registers that hold the sums, where a lane's row is one of four, and converted before the
// turn through LDS, which then moves 4, 2 or 1 bytes an output.  (Turned around as 32-bit sums, with the rows' parts read from LDS for eight columns at a time, as
// the feed-forward operators do: 4096 x 50257 x 2048 to E5M2 754 us.)
// UNIFORM: one factor for all.
template <int OUT, int NB, bool UNIFORM>
__device__ __forceinline__ void loss_store_gradient(v16f (&acc)[NB][4], uint8_t* smem, const LossArgs& o, void* D, int M, int N, int m0, int n0, int w)
{
    constexpr bool FP8OUT = OUT == OUT_E4M3 || OUT == OUT_E5M2;
    constexpr int FMT = OUT == OUT_E5M2 ? FP8_E5M2 : FP8_E4M3, ESZ = OUT == OUT_F32 ? 4 : OUT == OUT_BF16 ? 2 : 1;
    constexpr int WN = 32 * NB, ROWB = WN * ESZ + 16, LANES = WN * ESZ / 16, ROWS = 64 / LANES;      // of the turned block: bytes of a row, its lanes, rows a store
    static_assert(4 * 32 * ROWB <= OP_ROW_FACTORS && 64 % LANES == 0 && 32 % ROWS == 0, "room for the turned rows; whole rows");
    const int l = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));      // (see store_tile)
    const int h = l >> 5, wave_m0 = m0 + (w >> 1) * 128, wave_n0 = n0 + (w & 1) * WN;
    const bool n_edge = wave_n0 + WN > N;
    const double a_all = o.a_per_row ? 1.0 : 1.0 / (double)op_scalar(o.sA_dev), b_all = o.b_factors == B_ONE ? 1.0 / (double)op_scalar(o.sB_dev) : 1.0;
    const float f2 = (float)(a_all * b_all * (double)kLog2e);
    double* columns = (double*)(smem + OP_COLUMN_FACTORS) + w * 128;
    if (!UNIFORM && o.b_factors != B_ONE) {
#pragma unroll
        for (int i = 0; i < (NB + 1) / 2; ++i)
            if (64 * i + l < WN) *LDS_PTR(double, columns + 64 * i + l) = 1.0 / (double)o.sB_dev[min(wave_n0 + 64 * i + l, N - 1)];
    }
    // FP8 outputs: y sD with sD in the rows' parts, and the maximum divided by it at the end (4096 x 50257 x 2048 762 -> 751 us); where a part could overflow, or a
    // small maximum be lost (an exponential is 2^-126 or more, or 0), the outputs are multiplied one by one, on the way that also takes what has to be clamped: 815 us.
    // (As an instance of its own it would cost the other 765.)
    const float sD = FP8OUT && o.sD_dev ? op_scalar(o.sD_dev) : 1.0f;
    const bool large = __builtin_fabsf(sD) >= 1.0f;
    auto holds = [&](float x) __attribute__((always_inline)) {
        const float y = __builtin_fabsf(x * sD);
        return y < __builtin_inff() && (large || y >= 1.0f || x == 0.0f);
    };
    bool inside = true;
    if (FP8OUT) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const v4f part = *LDS_PTR(v4f, smem + OP_ROW_FACTORS + ((w >> 1) * 128 + 64 * i + l) * 16);
            inside &= (int)as_u32(part[3]) == -1 || (holds(part[1]) && holds(part[2]));
        }
    }
    const bool folded = FP8OUT && sD != 0.0f && __builtin_fabsf(sD) < __builtin_inff() && __all(inside);
    const float fold = folded ? sD : 1.0f, limit = !folded ? -1.0f : FMT == FP8_E4M3 ? 448.0f : 57344.0f;
    uint8_t* blk = smem + w * (32 * ROWB);
    uint8_t* d_wave = (uint8_t*)D + ((size_t)wave_m0 * N + wave_n0) * ESZ;
    const int st_row = l / LANES, st_col = (l % LANES) * 16, left = N - (wave_n0 + st_col / ESZ);
    unsigned top = 0;
#pragma unroll
    for (int mb = 0; mb < 4; ++mb) {
        const v4f part = *LDS_PTR(v4f, smem + OP_ROW_FACTORS + ((w >> 1) * 128 + 32 * mb + (l & 31)) * 16);
        const int row = wave_m0 + mb * 32 + (l & 31), column = (int)as_u32(part[3]);
        const bool none = column == -1;
        // (of a row without a label 2^-infinity times 0; what is infinite or NaN itself is taken out below)
        const float nlse2 = none ? -__builtin_inff() : -part[0], scale = none ? 0.0f : FP8OUT ? part[1] * fold : part[1];
        const float dloss = FP8OUT ? part[2] * fold : part[2];
        const int label = column >= wave_n0 && column < wave_n0 + WN ? column - wave_n0 : -1;
        float x[NB * 16];
#pragma unroll
        for (int i = 0; i < NB * 16; ++i) x[i] = acc[i >> 4][mb][i & 15];
        if (!UNIFORM) {
            const double fa = o.a_per_row ? 1.0 / (double)o.sA_dev[min(row, M - 1)] : a_all;
#pragma unroll
            for (int i = 0; i < NB * 16; ++i) x[i] *= (float)(fa * (o.b_factors == B_ONE ? b_all : *LDS_PTR(double, columns + loss_column(i, h))));
        }
        unsigned row_top = 0;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            float y[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[nb * 16 + i], UNIFORM ? f2 : kLog2e, nlse2)) * scale;
            if (__any(label >> 5 == nb)) {
#pragma unroll
                for (int i = 0; i < 16; ++i) y[i] = label == loss_column(nb * 16 + i, h) ? y[i] - dloss : y[i];
            }
            unsigned most = max_bits_of<16>(y);
            if (__any(none && most != 0)) {
#pragma unroll
                for (int i = 0; i < 16; ++i) y[i] = none ? 0.0f : y[i];
                most = none ? 0u : most;
            }
            if (n_edge && o.amax_out) {
#pragma unroll
                for (int i = 0; i < 16; ++i) row_top = max(row_top, wave_n0 + loss_column(nb * 16 + i, h) < N ? as_u32(y[i]) & 0x7fffffffu : 0u);
            } else {
                row_top = max(row_top, most);
            }
            uint8_t* dst = blk + (l & 31) * ROWB + (nb * 32 + 4 * h) * ESZ;
            if (OUT == OUT_F32) {
#pragma unroll
                for (int q = 0; q < 4; ++q) *LDS_PTR(v4f, dst + 8 * q * ESZ) = (v4f){y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]};
            } else if (OUT == OUT_BF16) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    v2i p;
                    p.x = (int)__builtin_bit_cast(unsigned, __builtin_convertvector((v2f){y[4 * q], y[4 * q + 1]}, v2bf));
                    p.y = (int)__builtin_bit_cast(unsigned, __builtin_convertvector((v2f){y[4 * q + 2], y[4 * q + 3]}, v2bf));
                    *LDS_PTR(v2i, dst + 8 * q * ESZ) = p;
                }
            } else {
                // (as in the plain epilogue: the largest value tells whether anything has to be clamped or looked at)
                u32x4 p;
                if (__all(as_f32(most) <= limit)) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) p[q] = encode4_inside<FMT>(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
                } else {
                    if (!folded) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) y[i] *= sD;
                    }
                    p = encode16<FMT, kCastCvt>(y);
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) *LDS_PTR(unsigned, dst + 8 * q) = p[q];
            }
        }
        if (row < M) top = max(top, row_top);
#pragma unroll
        for (int i = 0; i < 32 / ROWS; ++i) {
            const int r = i * ROWS + st_row;
            if (wave_m0 + mb * 32 + r >= M || left <= 0) continue;                         // beyond the edges of D
            uint8_t* out = d_wave + (size_t)(mb * 32 + r) * N * ESZ + st_col;
            const u32x4 p = *LDS_PTR(u32x4, blk + r * ROWB + st_col);
            if (left >= 16 / ESZ) {
                __builtin_nontemporal_store(p, (u32x4_any*)out);
            } else {                                        // the end of a row inside the lane's 16 bytes
#pragma unroll
                for (int e = 0; e < 16 / ESZ - 1; ++e) {
                    if (e < left) {
                        if (ESZ == 4) ((unsigned*)out)[e] = p[e & 3];
                        else if (ESZ == 2) ((unsigned short*)out)[e] = (unsigned short)(p[(e >> 1) & 3] >> (16 * (e & 1)));
                        else out[e] = (uint8_t)(p[e >> 2] >> (8 * (e & 3)));
                    }
                }
            }
        }
    }
    if (o.amax_out) {
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, d, 64));
        unsigned* cells = (unsigned*)(smem + OP_AMAX);
        if (l == 0) *LDS_PTR(unsigned, cells + w) = folded ? as_u32(__builtin_fabsf(as_f32(top) / sD)) : top;
        __syncthreads();
        // (unasked: 256 workgroups that end together queue up for a look at the cell longer than for the atomic itself, whose end nobody waits for)
        if (w == 0 && l == 0) {
            const u32x4 all = *LDS_PTR(u32x4, cells);
            atomicMax((unsigned*)o.amax_out, max(max(all[0], all[1]), max(all[2], all[3])));
        }
    }
}

template <int OUT, int NB>
__device__ __forceinline__ void loss_store_gradient(v16f (&acc)[NB][4], uint8_t* smem, const LossArgs& o, void* D, int M, int N, int m0, int n0, int w)
{
    if (!o.a_per_row && o.b_factors == B_ONE) loss_store_gradient<OUT, NB, true>(acc, smem, o, D, M, N, m0, n0, w);
    else loss_store_gradient<OUT, NB, false>(acc, smem, o, D, M, N, m0, n0, w);
}

// OP of the tile: 4 the loss, 5 its gradient.
template <int NB, int OP>
__device__ __forceinline__ void loss_store_tile(v16f (&acc)[NB][4], uint8_t* smem, const LossArgs& o, const LossRows<OP>& rows, void* D, int M, int N, int m0, int n0, int w)
{
    rows.leave(o, N, smem, w);
    if constexpr (OP == 4) loss_store_pairs<NB>(acc, smem, o, M, N, m0, n0, w);
    else switch (o.out_kind) {
        case OUT_F32: loss_store_gradient<OUT_F32, NB>(acc, smem, o, D, M, N, m0, n0, w); break;
        case OUT_BF16: loss_store_gradient<OUT_BF16, NB>(acc, smem, o, D, M, N, m0, n0, w); break;
        case OUT_E4M3: loss_store_gradient<OUT_E4M3, NB>(acc, smem, o, D, M, N, m0, n0, w); break;
        default: loss_store_gradient<OUT_E5M2, NB>(acc, smem, o, D, M, N, m0, n0, w); break;
    }
}

}  // namespace
}  // namespace fp8mm
