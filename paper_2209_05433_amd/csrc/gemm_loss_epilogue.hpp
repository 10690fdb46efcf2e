// How a workgroup of four waves that owns 256 rows x 64 NB columns of the logits leaves them (gemm_loss.hpp; gfx950): each wave 128 x 32 NB, as NB x 4 blocks of
// 32 x 32.
#pragma once

#include "gemm_loss.hpp"
#include "gemm_op_epilogue.hpp"

namespace fp8mm {
namespace {

// The loss: straight from the registers.  A lane holds half of a row's columns in each of its four rows (lane l and l + 32 the two halves), so a
// row's pair over the wave's columns takes one exchange between lanes, and no logit goes through LDS.
template <int NB>
__device__ __forceinline__ void loss_store_pairs(v16f (&acc)[NB][4], uint8_t* smem, const LossArgs& o, int M, int N, int m0, int n0, int w)
{
    const int l = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));      // (see store_tile)
    const int h = l >> 5, wave_m0 = m0 + (w >> 1) * 128, wave_n0 = n0 + (w & 1) * (32 * NB);
    if (wave_n0 >= N) return;
    const bool inside = wave_n0 + 32 * NB <= N, uniform = !o.a_per_row && o.b_factors == B_ONE;
    const double a_all = o.a_per_row ? 1.0 : 1.0 / (double)op_scalar(o.sA_dev), b_all = o.b_factors == B_ONE ? 1.0 / (double)op_scalar(o.sB_dev) : 1.0;
    double* columns = (double*)(smem + OP_COLUMN_FACTORS) + w * 128;
    if (o.b_factors != B_ONE) {
#pragma unroll
        for (int i = 0; i < (NB + 1) / 2; ++i)
            if (64 * i + l < 32 * NB) *LDS_PTR(double, columns + 64 * i + l) = 1.0 / (double)o.sB_dev[min(wave_n0 + 64 * i + l, N - 1)];
    }
    // narrow tiles behind wide ones (both widths in one launch) have two blocks of columns where a wide one has one
    const int64_t block = NB == 4 ? wave_n0 / 128 : wave_n0 / 64 - 2 * o.wide_cols;
    LossPair* pairs = (LossPair*)o.partials + block * M;
    float* targets = loss_targets(o, M, N);
    const float f = (float)(a_all * b_all), f2 = (float)(a_all * b_all * (double)kLog2e);
    auto row_block = [&](auto tag) __attribute__((always_inline)) {
        constexpr int MB = decltype(tag)::value;
        const int row = wave_m0 + 32 * MB + (l & 31), at = min(row, M - 1);
        const int64_t label = label_column(o, at) - wave_n0;
        const double fa = o.a_per_row ? 1.0 / (double)o.sA_dev[at] : a_all * b_all;
        float t[NB * 16];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 16; ++e) t[nb * 16 + e] = acc[nb][MB][e];
        if (!uniform) {
#pragma unroll
            for (int i = 0; i < NB * 16; ++i) {
                const int c = (i >> 4) * 32 + ((i >> 2) & 3) * 8 + 4 * h + (i & 3);
                const double fb = o.b_factors == B_ONE ? (o.a_per_row ? b_all : 1.0) : *LDS_PTR(double, columns + c);
                t[i] *= (float)((o.a_per_row || o.b_factors == B_ONE ? fa : a_all) * fb);
            }
        }
        // the label's column is in few of the tiles: its logit, from the same factor
        if (__any(label >= 0 && label < 32 * NB)) {
            float z = 0.0f;
#pragma unroll
            for (int i = 0; i < NB * 16; ++i) z = label == (i >> 4) * 32 + ((i >> 2) & 3) * 8 + 4 * h + (i & 3) ? t[i] : z;
            if (label >= 0 && label < 32 * NB && wave_n0 + label < N && ((label >> 2) & 1) == h && row < M) targets[row] = uniform ? z * f : z;
        }
        const float g = uniform ? f2 : kLog2e;
#pragma unroll
        for (int i = 0; i < NB * 16; ++i) t[i] *= g;
        if (!inside) {
#pragma unroll
            for (int i = 0; i < NB * 16; ++i) t[i] = wave_n0 + (i >> 4) * 32 + ((i >> 2) & 3) * 8 + 4 * h + (i & 3) < N ? t[i] : -__builtin_inff();
        }
        const LossPair p = loss_pair<NB * 16, 2, 32>(t);
        if (l < 32 && row < M) pairs[row] = p;
    };
    row_block(std::integral_constant<int, 0>{});
    row_block(std::integral_constant<int, 1>{});
    row_block(std::integral_constant<int, 2>{});
    row_block(std::integral_constant<int, 3>{});
}

// The gradient: turned around through LDS as by op_store_rows, behind which a lane has eight columns of a row; the rows' parts (LossRow) lie in LDS.
template <int NB>
__device__ __forceinline__ void loss_store_gradient(v16f (&acc)[NB][4], uint8_t* smem, const LossArgs& o, void* D, int M, int N, int m0, int n0, int w)
{
    constexpr int WN = 32 * NB, ROWB = WN * 4 + 16, MBS = NB == 4 ? 1 : 2, LANES = WN / 8, ROWS = 64 / LANES, G = 4;
    constexpr int STEPS = 32 * MBS / (ROWS * G), TURNS = 4 / MBS;
    static_assert(4 * 32 * MBS * ROWB <= OP_RING && OP_RING + 4 * 128 * 16 <= OP_ROW_FACTORS, "room for the turned rows and the rows' parts");
    const int l = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));      // (see store_tile)
    const int h = l >> 5;
    const int wave_m0 = m0 + (w >> 1) * 128, wave_n0 = n0 + (w & 1) * WN;
    const int col = wave_n0 + (l % LANES) * 8, left = N - col;
    uint8_t* blk = smem + w * (32 * MBS * ROWB);
    uint8_t* parts = smem + OP_RING + w * (128 * 16);
    double* row_factors = (double*)(smem + OP_ROW_FACTORS) + w * 128;
    double* column_factors = (double*)(smem + OP_COLUMN_FACTORS) + w * 128 + (l % LANES) * 8;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const LossRow r = loss_row(o, min(wave_m0 + 64 * i + l, M - 1));
        const int label = r.label >= 0 && r.label < N ? (int)r.label : r.label == -1 ? -1 : -2;
        *LDS_PTR(v4f, parts + (64 * i + l) * 16) = (v4f){-r.lse2, r.scale, r.dloss, as_f32((unsigned)label)};
        if (o.a_per_row) *LDS_PTR(double, row_factors + 64 * i + l) = 1.0 / (double)o.sA_dev[min(wave_m0 + 64 * i + l, M - 1)];
    }
    float f[8];
    {
        const double a_all = o.a_per_row ? 1.0 : 1.0 / (double)op_scalar(o.sA_dev);
        const bool one = o.b_factors == B_ONE;
        const double b_all = one ? 1.0 / (double)op_scalar(o.sB_dev) : 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double y = (one ? b_all : op_column_factor(o, N, min(col + i, N - 1), false)) * (double)kLog2e;
            f[i] = (float)(a_all * y);
            if (o.a_per_row) *LDS_PTR(double, column_factors + i) = y;
        }
    }
    const float sD = o.out_kind >= OUT_E4M3 && o.sD_dev ? op_scalar(o.sD_dev) : 1.0f;
    const bool inside = wave_m0 + 128 <= M && wave_n0 + WN <= N;
    unsigned top = 0;
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
            float x[G * 8], scale[G], dloss[G];
            int label[G];
            OutRows<G> t;
            t.col = col; t.left = left; t.rows = 0; t.whole = inside;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int in_wave = (i * G + g) * ROWS + l / LANES, row = wave_m0 + in_wave;
                const uint8_t* src = blk + ((in_turn * G + g) * ROWS + l / LANES) * ROWB + (l % LANES) * 32;
                const v4f part = *LDS_PTR(v4f, parts + in_wave * 16);
                scale[g] = part[1]; dloss[g] = part[2]; label[g] = (int)as_u32(part[3]);
                const double fa = o.a_per_row ? *LDS_PTR(double, row_factors + in_wave) : 1.0;
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const v4f s = *LDS_PTR(v4f, src + 16 * p);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float factor = o.a_per_row ? (float)(fa * *LDS_PTR(double, column_factors + 4 * p + e)) : f[4 * p + e];
                        x[8 * g + 4 * p + e] = __builtin_fmaf(s[e], factor, part[0]);
                    }
                }
                t.row[g] = row;
                if (row < M && left > 0) t.rows |= 1u << g;
            }
            top = max(top, loss_grad_finish<G, 8>(o, D, N, t, x, scale, dloss, label, sD));
        }
    }
    if (o.amax_out) {
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, d, 64));
        unsigned* cells = (unsigned*)(smem + OP_AMAX);
        if (l == 0) *LDS_PTR(unsigned, cells + w) = top;
        __syncthreads();
        if (w == 0) op_commit_top(o, l < 4 ? *LDS_PTR(unsigned, cells + l) : 0u);
    }
}

// OP of the tile: 4 the loss, 5 its gradient.
template <int NB, int OP>
__device__ __forceinline__ void loss_store_tile(v16f (&acc)[NB][4], uint8_t* smem, const LossArgs& o, void* D, int M, int N, int m0, int n0, int w)
{
    if constexpr (OP == 4) loss_store_pairs<NB>(acc, smem, o, M, N, m0, n0, w);
    else loss_store_gradient<NB>(acc, smem, o, D, M, N, m0, n0, w);
}

}  // namespace
}  // namespace fp8mm
