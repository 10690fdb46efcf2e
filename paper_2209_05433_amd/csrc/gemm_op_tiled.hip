// Products with an operator behind them on the tiles of the plain product (gemm_tile_body.hpp), for gfx950 (MI355X): 256 rows by 256 or 128
// columns of op(B), of the gated block 128 or 64 outputs with two columns of op(B) each.
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

template <int FA, int FB, int NB, int OP>
int launch_one(const GemmArgs& g, const OpArgs& o)
{
    constexpr bool A_KC = (FP8MM_LAYOUT & 2) == 0, B_KC = (FP8MM_LAYOUT & 1) != 0;
    constexpr int WIDTH = 64 * NB / (OP == 2 ? 2 : 1);
    static std::atomic<unsigned long long> attr_set{0ull};
    auto kern = gemm_op_tiled_kernel<FA, FB, FP8MM_ACC, A_KC, B_KC, NB, OP>;
    if (int e = raise_lds_limit((const void*)kern, FAST_LDS, attr_set)) return e;
    const int64_t tiles = ((g.M + BM - 1) / BM) * ((g.N + WIDTH - 1) / WIDTH);
    const int group = knob(FP8_KNOB_GROUP_M);
    enqueue(kern, dim3((unsigned)tiles), dim3(FAST_THREADS), FAST_LDS, g.stream, g.A, g.B, g.C, (int)g.M, (int)g.N, (int)g.K, o, group > 0 ? group : GROUP_M);
    return check_launch("gemm with an operator (tiled kernel)");
}

template <int FA, int FB>
int launch_formats(const GemmArgs& g, const OpArgs& o)
{
    if (op_pair_in(o.op)) return g.tile_n == 128 ? launch_one<FA, FB, 2, 2>(g, o) : launch_one<FA, FB, 4, 2>(g, o);
    return g.tile_n == 128 ? launch_one<FA, FB, 2, 1>(g, o) : launch_one<FA, FB, 4, 1>(g, o);
}

}  // namespace

#if !defined(FP8MM_LAYOUT) || !defined(FP8MM_ACC)
#error "compile with -DFP8MM_LAYOUT=0..3 (2 * transA + transB) and -DFP8MM_ACC=0|1"
#endif

int FP8MM_OP_TILED_NAME(FP8MM_LAYOUT, FP8MM_ACC)(const GemmArgs& g, const OpArgs& o)
{
    if (g.fmtA == FP8_E4M3)
        return g.fmtB == FP8_E4M3 ? launch_formats<FP8_E4M3, FP8_E4M3>(g, o) : launch_formats<FP8_E4M3, FP8_E5M2>(g, o);
    return g.fmtB == FP8_E4M3 ? launch_formats<FP8_E5M2, FP8_E4M3>(g, o) : launch_formats<FP8_E5M2, FP8_E5M2>(g, o);
}

}  // namespace fp8mm
