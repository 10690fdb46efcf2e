// Products with an operator behind them (gemm_op.hpp): which kernel takes a call, the kernel of plain FMAs that takes any, and the sum
// of the partial column sums (gfx950).
#include "gemm_op.hpp"

#include <algorithm>

namespace fp8mm {
namespace {

// ------------------------------------------------------------------------------------------
// Any shape, any alignment, every storage order: 64 x 64 outputs per workgroup of 256, 4 x 4 per thread, operands decoded to
// 32 bits (exactly) on their way into LDS, 32-bit FMAs.  The cross-check of the matrix-core forms, and what is left for the calls that they
// do not take.
// ------------------------------------------------------------------------------------------
constexpr int GT = 64, GK = 16;

template <int FMT_A, int FMT_B, bool PAIR>
__global__ __launch_bounds__(256) void gemm_op_generic_kernel(const uint8_t* __restrict__ A, const uint8_t* __restrict__ B, void* D,
                                                              int64_t M, int64_t N, int64_t K, OpArgs o, bool transA, bool transB)
{
    constexpr int P = PAIR ? 2 : 1;
    __shared__ float As[GK][GT + 1];
    __shared__ float Bs[P][GK][GT + 1];
    __shared__ float sums[16][GT];
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int64_t tiles_n = (N + GT - 1) / GT;
    const int64_t tm = blockIdx.x / tiles_n, m0 = tm * GT, n0 = (int64_t)(blockIdx.x % tiles_n) * GT;
    float acc[P][4][4] = {};
    for (int64_t k0 = 0; k0 < K; k0 += GK) {
        for (int e = tid; e < GT * GK; e += 256) {
            const int r = transA ? e % GT : e / GK, kk = transA ? e / GT : e % GK;      // consecutive lanes along the rows in memory
            const int64_t gm = m0 + r, gk = k0 + kk;
            As[kk][r] = gm < M && gk < K ? decode_fp8<FMT_A>(A[transA ? gk * M + gm : gm * K + gk]) : 0.0f;
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
            for (int e = tid; e < GT * GK; e += 256) {
                const int r = transB ? e / GK : e % GT, kk = transB ? e % GK : e / GT;
                const int64_t gn = n0 + r, gk = k0 + kk, at = gn + p * N;
                Bs[p][kk][r] = gn < N && gk < K ? decode_fp8<FMT_B>(B[transB ? at * K + gk : gk * (P * N) + at]) : 0.0f;
            }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < GK; ++kk)
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[p][i][j] = __builtin_fmaf(As[kk][ty * 4 + i], Bs[p][kk][tx * 4 + j], acc[p][i][j]);
        __syncthreads();
    }
    const float sD = o.out_kind >= OUT_E4M3 ? scale_value(o.sD_dev, 1.0f) : 1.0f;
    const int64_t col = n0 + tx * 4;
    const int left = col < N ? (int)(N - col < 4 ? N - col : 4) : 0;
    unsigned top = 0;
    float total[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (left > 0) {
        float bias[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (o.bias) load_row<4>(o.bias, o.bias_dtype, col, left, bias);
        double fy[4], fu[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t c = j < left ? col + j : col;
            fy[j] = op_column_factor(o, N, c, false);
            fu[j] = PAIR ? op_column_factor(o, N, c, true) : 0.0;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t row = m0 + ty * 4 + i;
            if (row >= M) continue;
            const double a = 1.0 / (double)o.sA_dev[o.a_per_row ? row : 0];
            float y[4], u[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                y[j] = acc[0][i][j] * (float)(a * fy[j]);
                u[j] = PAIR ? acc[P - 1][i][j] * (float)(a * fu[j]) : 0.0f;
            }
            top = max(top, op_row<4, PAIR>(o, D, N, row, col, left, y, u, bias, sD));
#pragma unroll
            for (int j = 0; j < 4; ++j) total[j] += y[j];
        }
    }
    if (o.sums) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sums[ty][tx * 4 + j] = total[j];
        __syncthreads();
        if (tid < GT && n0 + tid < N) {
            float s = 0.0f;
            for (int i = 0; i < 16; ++i) s += sums[i][tid];
            o.sums[tm * N + n0 + tid] = s;
        }
    }
    if (o.amax_out) {
        __shared__ unsigned tops[4];
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, d, 64));
        if ((tid & 63) == 0) tops[tid >> 6] = top;
        __syncthreads();
        if (tid < 64) op_commit_top(o, tid < 4 ? tops[tid] : 0u);
    }
}

template <int FA, int FB>
void enqueue_generic(const GemmArgs& g, const OpArgs& o, unsigned tiles)
{
    if (op_pair_in(o.op)) enqueue(gemm_op_generic_kernel<FA, FB, true>, dim3(tiles), dim3(256), 0, g.stream, g.A, g.B, g.C, g.M, g.N, g.K, o, g.transA, g.transB);
    else enqueue(gemm_op_generic_kernel<FA, FB, false>, dim3(tiles), dim3(256), 0, g.stream, g.A, g.B, g.C, g.M, g.N, g.K, o, g.transA, g.transB);
}

int launch_generic(const GemmArgs& g, const OpArgs& o)
{
    const int64_t tiles = ((g.M + GT - 1) / GT) * ((g.N + GT - 1) / GT);
    if (tiles > 0x7fffffffll) return fail(FP8_ERR_UNSUPPORTED, "gemm with an operator: %lld tiles of 64 x 64 exceed the grid limit", (long long)tiles);
    if (g.fmtA == FP8_E4M3) {
        if (g.fmtB == FP8_E4M3) enqueue_generic<FP8_E4M3, FP8_E4M3>(g, o, (unsigned)tiles);
        else enqueue_generic<FP8_E4M3, FP8_E5M2>(g, o, (unsigned)tiles);
    } else {
        if (g.fmtB == FP8_E4M3) enqueue_generic<FP8_E5M2, FP8_E4M3>(g, o, (unsigned)tiles);
        else enqueue_generic<FP8_E5M2, FP8_E5M2>(g, o, (unsigned)tiles);
    }
    return check_launch("gemm with an operator (plain FMAs)");
}

__global__ void op_zero_cell_kernel(unsigned* p) { *p = 0u; }

// dbias_j = sum of the rows of partial sums, always in the same order: a workgroup of 4 waves takes 64 columns, wave w the rows w, w + 4, ...
// No rows: zeros.  The workgroup behind the last columns reduces the maxima of the product's workgroups, where those are left in memory.
__global__ __launch_bounds__(256) void column_sum_kernel(const float* __restrict__ sums, int64_t parts, int64_t N, float* __restrict__ dbias,
                                                         const unsigned* __restrict__ tops, unsigned ntops, unsigned* __restrict__ amax_out)
{
    __shared__ float part[4][64];
    const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t col = (int64_t)blockIdx.x * 64 + l;
    if (tops && blockIdx.x == gridDim.x - 1) {
        unsigned m = 0;
        for (unsigned i = threadIdx.x; i < ntops; i += 256) m = max(m, tops[i]);
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) m = max(m, (unsigned)__shfl_xor((int)m, d, 64));
        if (l == 0) part[w][0] = as_f32(m);
        __syncthreads();
        if (threadIdx.x == 0) *amax_out = max(max(as_u32(part[0][0]), as_u32(part[1][0])), max(as_u32(part[2][0]), as_u32(part[3][0])));
        return;
    }
    float s = 0.0f;
    if (col < N)
        for (int64_t i = w; i < parts; i += 4) s += sums[i * N + col];
    part[w][l] = s;
    __syncthreads();
    if (w == 0 && col < N) dbias[col] = (part[0][l] + part[1][l]) + (part[2][l] + part[3][l]);
}

// Which kernel takes the call: the one of few rows where it pays, else what the plain product of the same operands takes, as far as it exists with these ends
// (not the any-shape kernel, tiles of 192 columns or the persistent form).
struct OpPlan { bool generic, tiled; int small, acc, tile_n, wide_cols; bool skinny; };
OpPlan plan_op(const GemmArgs& g, const OpArgs& o)
{
    const bool pair = op_pair_in(o.op);
    const OpPlan plain_fmas = {true, false, SMALL_NONE, 0, 0, 0, false};
    GemmArgs p = g;
    if (pair) p.N = 2 * g.N;
    p.ep = o;
    p.ep.b_per_col = o.b_factors != B_ONE;
    if (g.K == 0 || (pair && !g.transB && g.N < 16)) return plain_fmas;
    const bool chosen = !knob(FP8_KNOB_SMALL) && !knob(FP8_KNOB_GEMM_KERNEL) && !knob(FP8_KNOB_TILE_N);      // no knob asks for another kernel
    if (chosen && op_skinny_takes(g, pair)) return {false, false, SMALL_NONE, (int)ACC_F16, 0, 0, true};
    const GemmPlan plan = plan_gemm(p, false);
    if (plan.kernel == GEMM_GENERIC) return plain_fmas;
    // Shapes and alignments outside the tiled kernel's, and any K that is no multiple of 16, are computed on the fp16 instructions, whatever the flag
    // says: callers are promised fp8_gemm's bound there.  (Of a gated block F is what has to be a multiple of 16, not 2 F.)
    const bool halves = !pair || g.transB || g.N % 16 == 0;
    const int acc = plan.kernel == GEMM_MFMA_ANY || !halves || g.K % 16 ? (int)ACC_F16 : g.acc;
    if (plan.small != SMALL_NONE) return {false, false, plan.small, acc, 0, 0, false};
    // The tiled kernel exists for a weight in E4M3 (the format of weights); E5M2, and shapes and alignments that it does not take, go to tiles of 64 x 64 (4096 x 6144 x
    // 2048 with GELU 108 us, in E5M2 171; with K = 2047 226; up to some hundreds of tiles as fast as the plain product).
    const bool tiled = plan.kernel != GEMM_MFMA_ANY && g.fmtB == FP8_E4M3 && halves && (!pair || !g.transB || (uint64_t)(g.N + TILE_M) * (uint64_t)g.K < (1ull << 32));
    if (!tiled) return ((g.M + 63) / 64) * ((p.N + 63) / 64) > 0x7fffffffll ? plain_fmas : OpPlan{false, false, SMALL_64x64, acc, 0, 0, false};
    // The width whose rounds of 256 workgroups take less time, or both widths in one launch, by the plain product's model of run times with the
    // operator's own time on top (us of a 256-wide tile: fitted to 8192 x 8192 outputs over K = 256; it is the same per output in both widths).
    const TileTimes t = tile_times(acc, 2.0 * (double)((g.K + 2 * TILE_K - 1) / (2 * TILE_K)));
    const double own = o.op == OP_GATED_GRAD ? 25.0 : o.op == OP_GATED ? 3.0 : o.op == OP_ACT_GRAD || o.side ? 12.0 : 7.0;
    const double wide = t.wide + own, narrow = t.narrow + 0.5 * own;
    const int64_t tiles_m = (g.M + TILE_M - 1) / TILE_M, wide_all = (p.N + 255) / 256, narrow_all = (p.N + 127) / 128;
    const double us_wide = tiles_makespan(tiles_m * wide_all, 0, wide, narrow), us_narrow = tiles_makespan(0, tiles_m * narrow_all, wide, narrow);
    OpPlan r = {false, true, SMALL_NONE, acc, us_narrow < us_wide ? 128 : 256, 0, false};
    const int forced = knob(FP8_KNOB_TILE_N), mixed = knob(FP8_KNOB_MIXED);
    if (forced) r.tile_n = forced;
    if (forced || mixed == 1 || wide_all < 2) return r;
    if (mixed == 2) {
        r.wide_cols = (int)(wide_all / 2);
        return r;
    }
    // (as many wide columns as whole rounds hold: fewer or more leave units idle between the widths; beyond 16 rounds the last one matters little)
    double best = 0.97 * std::min(us_wide, us_narrow);
    for (int64_t units = 256; units / tiles_m < wide_all && tiles_m * wide_all <= 16 * 256; units += 256) {
        const int64_t c = std::max<int64_t>(units / tiles_m, 1);
        const double us = tiles_makespan(tiles_m * c, tiles_m * ((p.N - c * 256 + 127) / 128), wide, narrow) + 3.0;
        if (us < best) { best = us; r.wide_cols = (int)c; }
    }
    return r;
}

}  // namespace

int raise_lds_limit(const void* kernel, int bytes, std::atomic<unsigned long long>& done)
{
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return fail(FP8_ERR_DEVICE, "hipGetDevice failed");
    const unsigned long long bit = 1ull << (dev & 63);
    if (dev < 64 && (done.load(std::memory_order_relaxed) & bit)) return FP8_OK;
    const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return fail(FP8_ERR_DEVICE, "hipFuncSetAttribute(LDS=%d): %s", bytes, hipGetErrorString(e));
    if (dev < 64) done.fetch_or(bit, std::memory_order_relaxed);
    return FP8_OK;
}

int launch_gemm_op(const GemmArgs& g, const OpArgs& args, float* dbias)
{
    typedef int (*small_fn)(const GemmArgs&, const OpArgs&, int);
    static const small_fn small[4] = {FP8MM_OP_SMALL_NAME(0), FP8MM_OP_SMALL_NAME(1), FP8MM_OP_SMALL_NAME(2), FP8MM_OP_SMALL_NAME(3)};
    typedef int (*tiled_fn)(const GemmArgs&, const OpArgs&);
    static const tiled_fn tiled[4][2] = {{FP8MM_OP_TILED_NAME(0, 0), FP8MM_OP_TILED_NAME(0, 1)}, {FP8MM_OP_TILED_NAME(1, 0), FP8MM_OP_TILED_NAME(1, 1)},
                                         {FP8MM_OP_TILED_NAME(2, 0), FP8MM_OP_TILED_NAME(2, 1)}, {FP8MM_OP_TILED_NAME(3, 0), FP8MM_OP_TILED_NAME(3, 1)}};
    if (dbias && g.N > (int64_t)0x7fffffff * 32) return fail(FP8_ERR_UNSUPPORTED, "gemm with an operator: dbias of %lld values exceeds the grid limit", (long long)g.N);
    const bool work = g.M > 0 && g.N > 0;
    OpArgs o = args;
    OpPlan plan{};
    int64_t parts = 0, tops = 0;                             // rows of partial sums; workgroups that leave their maxima in memory
    if (work) {
        plan = plan_op(g, o);
        int64_t rows = 64, width = 64;                       // of a workgroup's outputs
        if (plan.skinny) { rows = 16; width = 16; }
        else if (plan.tiled) { rows = TILE_M; width = plan.tile_n; }
        else if (plan.small == SMALL_32x32 || plan.small == SMALL_32x64) { rows = 32; width = plan.small == SMALL_32x32 ? 32 : 64; }
        auto count = [](int64_t n, int64_t per) { return (n + per - 1) / per; };
        parts = count(g.M, plan.tiled ? rows / 2 : rows);
        if (o.sums && parts == 1) { o.sums = dbias; dbias = nullptr; }      // one row of partial sums is the sum
        // With a bias gradient there is a launch behind the product anyway: it takes the maxima along, if the workspace has room for them behind the
        // partial sums (4.5 us less than a cell that has to be cleared first).
        if (dbias && o.amax_out) {
            tops = count(g.M, rows) * (plan.wide_cols ? plan.wide_cols + count(g.N - plan.wide_cols * (int64_t)256, 128) : count(g.N, width));
            if ((count(g.M, kOpSumRows) - parts) * g.N >= tops && tops <= 0x7fffffff) o.tops = (unsigned*)(o.sums + parts * g.N);
        }
    }
    if (o.amax_out && !o.tops) {                             // written, not accumulated
        enqueue(op_zero_cell_kernel, dim3(1), dim3(1), 0, g.stream, (unsigned*)o.amax_out);
        if (int e = check_launch("gemm with an operator (amax init)")) return e;
    }
    if (work) {
        const int order = (g.transA ? 2 : 0) + (g.transB ? 1 : 0);
        GemmArgs p = g;
        p.acc = plan.acc; p.tile_n = plan.tile_n; p.wide_cols = plan.wide_cols;
        if (int e = plan.generic ? launch_generic(g, o) : plan.skinny ? launch_op_skinny(g, o) : plan.tiled ? tiled[order][plan.acc == ACC_FP8 ? 1 : 0](p, o)
                                                                                                            : small[order](p, o, plan.small)) return e;
    }
    if (dbias && g.N > 0) {
        enqueue(column_sum_kernel, dim3((unsigned)((g.N + 63) / 64) + (o.tops ? 1 : 0)), dim3(256), 0, g.stream, o.sums, parts, g.N, dbias, o.tops, (unsigned)tops,
                (unsigned*)o.amax_out);
        return check_launch("gemm with an operator (column sums)");
    }
    return FP8_OK;
}

}  // namespace fp8mm
