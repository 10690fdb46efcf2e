// How a workgroup of four waves that owns 256 rows x 64 NB columns of a product leaves them through an operator (gfx950): each wave 128 x 32 NB,
// as NB x 4 blocks of 32 x 32.
#pragma once

#include "gemm_epilogue.hpp"
#include "gemm_op.hpp"

namespace fp8mm {
namespace {

// A lane holds 4 consecutive columns of a row per accumulator quad.  As in the plain epilogue the wave turns 32 rows at a time around
// through its own piece of the idle LDS, here as the 32-bit sums: behind the turn a lane has 8 columns of a row, 8 (or 4) lanes a whole line of a
// 16-bit matrix, and everything else (factors, bias, the tensors that are read and kept, the activation) is done there, where every
// access to memory is 16 bytes a lane along the rows.  PAIR: the first half of the wave's columns are its outputs' gate, the other half the same
// outputs' second projection.  A lane's columns are the same in all rows: its bias and factors stay in registers, and so do
// its column sums, which meet the other lanes' of the wave's 128 rows at the end, in a fixed order.
template <int NB, bool PAIR>
__device__ __forceinline__ void op_store_tile(v16f (&acc)[NB][4], uint8_t* smem, const OpArgs& o, void* D, int M, int N, int m0, int n0, int w)
{
    constexpr int WN = 32 * NB, OUTW = PAIR ? WN / 2 : WN;      // columns of the wave, outputs of a row
    constexpr int ROWB = WN * 4 + 16;                           // padded LDS row
    constexpr int LANES = OUTW / 8, ROWS = 64 / LANES;          // lanes that hold a row between them, rows at a time
    static_assert(64 % LANES == 0, "whole rows");
    const int l = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));      // (see store_tile)
    const int h = l >> 5, wn = w & 1;
    const int wave_m0 = m0 + (w >> 1) * 128, wave_n0 = n0 + wn * OUTW;
    const int col = wave_n0 + (l % LANES) * 8, left = N - col;
    uint8_t* blk = smem + w * (32 * ROWB);

    // factors: one for both operands, or the reciprocals of the columns' (times that of A, where it has one), in 64 bits until the product is rounded
    double col_y[8], col_u[8];
    float fy[8], fu[8], bias[8];
    const double a_all = o.a_per_row ? 1.0 : 1.0 / (double)o.sA_dev[0];
    {
        const bool one = o.b_factors == B_ONE;
        const double b_all = one ? 1.0 / (double)o.sB_dev[0] : 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = min(col + i, N - 1);
            col_y[i] = one ? b_all : op_column_factor(o, N, c, false);
            col_u[i] = !PAIR ? 0.0 : one ? b_all : op_column_factor(o, N, c, true);
            fy[i] = (float)(a_all * col_y[i]);
            fu[i] = (float)(a_all * col_u[i]);
            bias[i] = 0.0f;
        }
        if (!PAIR && o.bias && left > 0) load_row<8>(o.bias, o.bias_dtype, col, left, bias);
    }
    const float sD = o.out_kind >= OUT_E4M3 ? scale_value(o.sD_dev, 1.0f) : 1.0f;
    float column[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    unsigned top = 0;
#pragma unroll
    for (int mb = 0; mb < 4; ++mb) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *LDS_PTR(v4f, blk + (l & 31) * ROWB + (nb * 32 + 8 * q + 4 * h) * 4) =
                    (v4f){acc[nb][mb][4 * q], acc[nb][mb][4 * q + 1], acc[nb][mb][4 * q + 2], acc[nb][mb][4 * q + 3]};
#pragma unroll 1
        for (int i = 0; i < 32 / ROWS; ++i) {
            const int r = i * ROWS + l / LANES, row = wave_m0 + mb * 32 + r;
            if (row >= M || left <= 0) continue;
            const uint8_t* src = blk + r * ROWB + (l % LANES) * 32;
            float y[8], u[8];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const v4f a = *LDS_PTR(v4f, src + 16 * j);
                v4f b = {0.0f, 0.0f, 0.0f, 0.0f};
                if (PAIR) b = *LDS_PTR(v4f, src + OUTW * 4 + 16 * j);
#pragma unroll
                for (int e = 0; e < 4; ++e) { y[4 * j + e] = a[e]; u[4 * j + e] = b[e]; }
            }
            if (o.a_per_row) {
                const double a = 1.0 / (double)o.sA_dev[row];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    fy[e] = (float)(a * col_y[e]);
                    if (PAIR) fu[e] = (float)(a * col_u[e]);
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y[e] *= fy[e];
                if (PAIR) u[e] *= fu[e];
            }
            top = max(top, op_row<8, PAIR>(o, D, N, row, col, left, y, u, bias, sD));
            if (!PAIR && o.sums) {
#pragma unroll
                for (int e = 0; e < 8; ++e) column[e] += y[e];
            }
        }
    }
    if (!PAIR && o.sums && wave_m0 < M) {
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
        unsigned* cells = (unsigned*)(smem + EP_AMAX);
        if (l == 0) *LDS_PTR(unsigned, cells + w) = top;
        __syncthreads();
        if (w == 0) wave_amax_commit(l < 4 ? *LDS_PTR(unsigned, cells + l) : 0u, o.amax_out);
    }
}

}  // namespace
}  // namespace fp8mm
