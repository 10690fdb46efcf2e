// Products with an operator behind them on the tiles of the plain product (gemm_tile_body.hpp), for gfx950 (MI355X): 256 rows by 256 or 128
// columns of op(B), of the gated block 128 or 64 outputs with two columns of op(B) each, or both widths in one launch.
//
// This file is compiled once per (storage orders, accumulation mode): -DFP8MM_LAYOUT, -DFP8MM_ACC.
#include "gemm_tile_body.hpp"

#include <atomic>

namespace fp8mm {
namespace {

template <int FMT_A, int FMT_B, int ACC, bool A_KC, bool B_KC, int NB, int OP>
__global__ __launch_bounds__(FAST_THREADS, 1) void gemm_op_tiled_kernel(const uint8_t* __restrict__ A, const uint8_t* __restrict__ B, void* D,
                                                                        int M, int N, int K, OpArgs o, int group_m)
{
    constexpr int WIDTH = 64 * NB / (OP == 2 ? 2 : 1);
    gemm_tile_body<FMT_A, FMT_B, ACC, A_KC, B_KC, NB, false, OP>(A, B, D, M, N, K, o, group_m, 1, (K + 2 * BK - 1) / (2 * BK), (int)blockIdx.x, 0,
                                                                 (N + WIDTH - 1) / WIDTH);
}

// The first wide_cols tile columns 256 columns of op(B) wide, the others 128, in one launch, the wide ones first (see gemm_tiled.hip).
template <int FMT_A, int FMT_B, int ACC, bool A_KC, bool B_KC, int OP>
__global__ __launch_bounds__(FAST_THREADS, 1) void gemm_op_mixed_kernel(const uint8_t* __restrict__ A, const uint8_t* __restrict__ B, void* D,
                                                                        int M, int N, int K, OpArgs o, int group_m, int wide_cols)
{
    constexpr int WIDE = OP == 2 ? 128 : 256, NARROW = WIDE / 2;          // output columns
    const int pairs = (K + 2 * BK - 1) / (2 * BK), wide_tiles = ((M + BM - 1) / BM) * wide_cols;
    if ((int)blockIdx.x < wide_tiles)
        gemm_tile_body<FMT_A, FMT_B, ACC, A_KC, B_KC, 4, false, OP>(A, B, D, M, N, K, o, group_m, 1, pairs, (int)blockIdx.x, 0, wide_cols);
    else
        gemm_tile_body<FMT_A, FMT_B, ACC, A_KC, B_KC, 2, false, OP>(A, B, D, M, N, K, o, group_m, 1, pairs, (int)blockIdx.x - wide_tiles, wide_cols * WIDE,
                                                                    (N - wide_cols * WIDE + NARROW - 1) / NARROW);
}

int group_m_setting()
{
    const int v = knob(FP8_KNOB_GROUP_M);
    return v > 0 ? v : GROUP_M;
}

template <int FA, int FB, int NB, int OP>
int launch_one(const GemmArgs& g, const OpArgs& o)
{
    constexpr bool A_KC = (FP8MM_LAYOUT & 2) == 0, B_KC = (FP8MM_LAYOUT & 1) != 0;
    constexpr int WIDTH = 64 * NB / (OP == 2 ? 2 : 1);
    static std::atomic<unsigned long long> attr_set{0ull};
    auto kern = gemm_op_tiled_kernel<FA, FB, FP8MM_ACC, A_KC, B_KC, NB, OP>;
    if (int e = raise_lds_limit((const void*)kern, FAST_LDS, attr_set)) return e;
    const int64_t tiles = ((g.M + BM - 1) / BM) * ((g.N + WIDTH - 1) / WIDTH);
    enqueue(kern, dim3((unsigned)tiles), dim3(FAST_THREADS), FAST_LDS, g.stream, g.A, g.B, g.C, (int)g.M, (int)g.N, (int)g.K, o, group_m_setting());
    return check_launch("gemm with an operator (tiled kernel)");
}

template <int FA, int FB, int OP>
int launch_mixed(const GemmArgs& g, const OpArgs& o)
{
    constexpr bool A_KC = (FP8MM_LAYOUT & 2) == 0, B_KC = (FP8MM_LAYOUT & 1) != 0;
    constexpr int WIDE = OP == 2 ? 128 : 256, NARROW = WIDE / 2;
    static std::atomic<unsigned long long> attr_set{0ull};
    auto kern = gemm_op_mixed_kernel<FA, FB, FP8MM_ACC, A_KC, B_KC, OP>;
    if (int e = raise_lds_limit((const void*)kern, FAST_LDS, attr_set)) return e;
    const int64_t tiles_m = (g.M + BM - 1) / BM, tiles = tiles_m * g.wide_cols + tiles_m * ((g.N - (int64_t)g.wide_cols * WIDE + NARROW - 1) / NARROW);
    enqueue(kern, dim3((unsigned)tiles), dim3(FAST_THREADS), FAST_LDS, g.stream, g.A, g.B, g.C, (int)g.M, (int)g.N, (int)g.K, o, group_m_setting(), g.wide_cols);
    return check_launch("gemm with an operator (tiled kernel, both tile widths)");
}

template <int FA, int FB, int OP>
int launch_width(const GemmArgs& g, const OpArgs& o)
{
    if (g.wide_cols > 0) return launch_mixed<FA, FB, OP>(g, o);
    return g.tile_n == 128 ? launch_one<FA, FB, 2, OP>(g, o) : launch_one<FA, FB, 4, OP>(g, o);
}

template <int FA>
int launch_op(const GemmArgs& g, const OpArgs& o)
{
    switch (o.op) {
        case OP_ACT: return launch_width<FA, FP8_E4M3, 1>(g, o);
        case OP_GATED: return launch_width<FA, FP8_E4M3, 2>(g, o);
        default: return launch_width<FA, FP8_E4M3, 3>(g, o);
    }
}

}  // namespace

#if !defined(FP8MM_LAYOUT) || !defined(FP8MM_ACC)
#error "compile with -DFP8MM_LAYOUT=0..3 (2 * transA + transB) and -DFP8MM_ACC=0|1"
#endif

int FP8MM_OP_TILED_NAME(FP8MM_LAYOUT, FP8MM_ACC)(const GemmArgs& g, const OpArgs& o)
{
    return g.fmtA == FP8_E4M3 ? launch_op<FP8_E4M3>(g, o) : launch_op<FP8_E5M2>(g, o);
}

}  // namespace fp8mm
