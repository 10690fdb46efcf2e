// Tiled FP8 x FP8 GEMM with fp32 accumulation and the fused epilogue, for gfx950 (MI355X): the kernels around the tile of
// gemm_tile_body.hpp, where the design is described.
//
// This file is compiled once per (storage orders, accumulation mode): -DFP8MM_LAYOUT, -DFP8MM_ACC.
#include "gemm_tile_body.hpp"

#include <atomic>
#include <type_traits>

namespace fp8mm {
namespace {

template <int FMT_A, int FMT_B, int ACC, bool A_KC, bool B_KC, int NB, bool PERSIST>
__global__ __launch_bounds__(FAST_THREADS, 1) void gemm_fast_kernel(
    const uint8_t* __restrict__ A, const uint8_t* __restrict__ B, void* __restrict__ C,
    int M, int N, int K, EpilogueArgs ep, int group_m, int splits, int pairs_per_split)
{
    gemm_tile_body<FMT_A, FMT_B, ACC, A_KC, B_KC, NB, PERSIST>(A, B, C, M, N, K, ep, group_m, splits, pairs_per_split,
                                                              (int)blockIdx.x, 0, (N + 64 * NB - 1) / (64 * NB));
}

// Two tile widths in one launch: the first wide_cols tile columns of the output in tiles of 256 x 64 NB (256 or
// 192 wide; workgroups 0 .. tiles_m * wide_cols - 1, dispatched first), the remaining columns in 256 x 128
// tiles.  For problems whose tiles of one width leave much of the last round of workgroups empty
// (4096 x 6144: 384 wide tiles = 1.5 rounds, 768 narrow ones = 3 rounds at 0.6 of the wide tile's
// time each; 256 wide + 256 narrow = one round of each); the narrow tiles also fill the compute
// units that the last wide tiles leave idle.  The choice of wide_cols is the dispatcher's.
template <int FMT_A, int FMT_B, int ACC, bool A_KC, bool B_KC, int NB>
__global__ __launch_bounds__(FAST_THREADS, 1) void gemm_mixed_kernel(
    const uint8_t* __restrict__ A, const uint8_t* __restrict__ B, void* __restrict__ C,
    int M, int N, int K, EpilogueArgs ep, int group_m, int pairs, int wide_cols)
{
    const int wide_tiles = ((M + BM - 1) / BM) * wide_cols;
    if ((int)blockIdx.x < wide_tiles)
        gemm_tile_body<FMT_A, FMT_B, ACC, A_KC, B_KC, NB, false>(A, B, C, M, N, K, ep, group_m, 1, pairs, (int)blockIdx.x, 0, wide_cols);
    else
        gemm_tile_body<FMT_A, FMT_B, ACC, A_KC, B_KC, 2, false>(A, B, C, M, N, K, ep, group_m, 1, pairs, (int)blockIdx.x - wide_tiles,
                                                                wide_cols * (64 * NB), (N - wide_cols * (64 * NB) + 127) / 128);
}

// ---- launch ------------------------------------------------------------------------------
// The knob FP8_KNOB_GROUP_M sets the number of tile rows per band of the tile order (0: GROUP_M).
int group_m_setting()
{
    const int v = knob(FP8_KNOB_GROUP_M);
    return v > 0 ? v : GROUP_M;
}

template <int FA, int FB, int ACC, bool A_KC, bool B_KC, int NB, bool PERSIST = false>
int launch_fast(const GemmArgs& g)
{
    // the kernel needs more dynamic LDS than the default limit: raised once per device
    static std::atomic<unsigned long long> attr_set{0ull};
    auto kern = gemm_fast_kernel<FA, FB, ACC, A_KC, B_KC, NB, PERSIST>;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return fail(FP8_ERR_DEVICE, "hipGetDevice failed");
    const unsigned long long bit = 1ull << (dev & 63);
    if (dev >= 64 || !(attr_set.load(std::memory_order_relaxed) & bit)) {
        hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, FAST_LDS);
        if (e != hipSuccess)
            return fail(FP8_ERR_DEVICE, "hipFuncSetAttribute(LDS=%d): %s", FAST_LDS, hipGetErrorString(e));
        if (dev < 64) attr_set.fetch_or(bit, std::memory_order_relaxed);
    }
    constexpr int BN = 64 * NB;
    const int tiles = (int)(((g.M + BM - 1) / BM) * ((g.N + BN - 1) / BN));
    const int pairs = (int)((g.K + 2 * BK - 1) / (2 * BK));
    const int splits = !PERSIST && g.splits > 1 ? g.splits : 1;
    const int grid = PERSIST ? min(tiles, compute_units()) : tiles * splits;
    enqueue(kern, dim3(grid), dim3(FAST_THREADS), FAST_LDS, g.stream, g.A, g.B, g.C,
                       (int)g.M, (int)g.N, (int)g.K, g.ep, group_m_setting(), splits,
                       splits > 1 ? g.pairs_per_split : pairs);
    return check_launch(PERSIST ? "gemm (tiled kernel, persistent form)" : "gemm (tiled kernel)");
}

template <int FA, int FB, int ACC, bool A_KC, bool B_KC, int NB>
int launch_mixed(const GemmArgs& g)
{
    static std::atomic<unsigned long long> attr_set{0ull};
    auto kern = gemm_mixed_kernel<FA, FB, ACC, A_KC, B_KC, NB>;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return fail(FP8_ERR_DEVICE, "hipGetDevice failed");
    const unsigned long long bit = 1ull << (dev & 63);
    if (dev >= 64 || !(attr_set.load(std::memory_order_relaxed) & bit)) {
        hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, FAST_LDS);
        if (e != hipSuccess)
            return fail(FP8_ERR_DEVICE, "hipFuncSetAttribute(LDS=%d): %s", FAST_LDS, hipGetErrorString(e));
        if (dev < 64) attr_set.fetch_or(bit, std::memory_order_relaxed);
    }
    const int64_t tiles_m = (g.M + BM - 1) / BM;
    const int64_t grid = tiles_m * g.wide_cols + tiles_m * ((g.N - (int64_t)g.wide_cols * (64 * NB) + 127) / 128);
    const int pairs = (int)((g.K + 2 * BK - 1) / (2 * BK));
    enqueue(kern, dim3((unsigned)grid), dim3(FAST_THREADS), FAST_LDS, g.stream, g.A, g.B, g.C,
                       (int)g.M, (int)g.N, (int)g.K, g.ep, group_m_setting(), pairs, g.wide_cols);
    return check_launch("gemm (tiled kernel, both tile widths)");
}

}  // namespace

#if !defined(FP8MM_LAYOUT) || !defined(FP8MM_ACC)
#error "compile with -DFP8MM_LAYOUT=0..3 (2 * transA + transB) and -DFP8MM_ACC=0|1"
#endif

template <int NB>
static int launch_formats(const GemmArgs& g)
{
    constexpr bool A_KC = (FP8MM_LAYOUT & 2) == 0;   // A row-major M x K is K-contiguous
    constexpr bool B_KC = (FP8MM_LAYOUT & 1) != 0;   // B stored N x K is K-contiguous
    constexpr int ACC = FP8MM_ACC;
    if (NB == 2 && g.persist) {                      // the persistent form exists for the narrow tile
        if (g.fmtA == FP8_E4M3)
            return g.fmtB == FP8_E4M3 ? launch_fast<FP8_E4M3, FP8_E4M3, ACC, A_KC, B_KC, 2, true>(g)
                                      : launch_fast<FP8_E4M3, FP8_E5M2, ACC, A_KC, B_KC, 2, true>(g);
        return g.fmtB == FP8_E4M3 ? launch_fast<FP8_E5M2, FP8_E4M3, ACC, A_KC, B_KC, 2, true>(g)
                                  : launch_fast<FP8_E5M2, FP8_E5M2, ACC, A_KC, B_KC, 2, true>(g);
    }
    if (g.fmtA == FP8_E4M3)
        return g.fmtB == FP8_E4M3 ? launch_fast<FP8_E4M3, FP8_E4M3, ACC, A_KC, B_KC, NB>(g)
                                  : launch_fast<FP8_E4M3, FP8_E5M2, ACC, A_KC, B_KC, NB>(g);
    return g.fmtB == FP8_E4M3 ? launch_fast<FP8_E5M2, FP8_E4M3, ACC, A_KC, B_KC, NB>(g)
                              : launch_fast<FP8_E5M2, FP8_E5M2, ACC, A_KC, B_KC, NB>(g);
}

template <int NB>
static int launch_mixed_formats(const GemmArgs& g)
{
    constexpr bool A_KC = (FP8MM_LAYOUT & 2) == 0, B_KC = (FP8MM_LAYOUT & 1) != 0;
    constexpr int ACC = FP8MM_ACC;
    if (g.fmtA == FP8_E4M3)
        return g.fmtB == FP8_E4M3 ? launch_mixed<FP8_E4M3, FP8_E4M3, ACC, A_KC, B_KC, NB>(g) : launch_mixed<FP8_E4M3, FP8_E5M2, ACC, A_KC, B_KC, NB>(g);
    return g.fmtB == FP8_E4M3 ? launch_mixed<FP8_E5M2, FP8_E4M3, ACC, A_KC, B_KC, NB>(g) : launch_mixed<FP8_E5M2, FP8_E5M2, ACC, A_KC, B_KC, NB>(g);
}

int FP8MM_TILED_NAME(FP8MM_LAYOUT, FP8MM_ACC)(const GemmArgs& g)
{
    if (g.wide_cols > 0) return g.tile_n == 192 ? launch_mixed_formats<3>(g) : launch_mixed_formats<4>(g);
    return g.tile_n == 128 ? launch_formats<2>(g) : g.tile_n == 192 ? launch_formats<3>(g) : launch_formats<4>(g);
}

}  // namespace fp8mm
