// Softmax cross entropy behind a product whose columns are a vocabulary (fp8_gemm_xent, fp8_gemm_xent_grad; gfx950): the arguments, a row's share of the
// sum, and the step from sums of products to the gradient.
//
//   z = acc / (sA_i sB_j);  lse_i = log sum_j e^z;  loss_i = lse_i - z_i,label + w lse_i^2;  y = dloss_i (e^(z - lse_i) (1 + 2 w lse_i) - [j is the label])
//
// Everything is in base 2: t = z log2(e), whose factor is folded into 1 / (sA sB), so that an exponential is one instruction.  A tile leaves for each of its rows
// the pair (ref, sum of 2^(t - ref)) over its columns, ref their largest t; loss_join_kernel adds up a row's pairs.  ref is held within the finite numbers: of a
// row whose logits are all -infinity every term is then 2^-infinity = 0 (and not 2^NaN), and +infinity makes the sum +infinity.
// No logit is ever stored: a row of a tile leaves 8 bytes where its logits are 128 to 512.
//
// Bound by the matrix cores (one exponential beside 2 K operations, a part of the tile's end): 8192 x 50257 x 12288 at 1.51 to 1.55 PFLOP/s, 87 % of the matrix cycles busy;
// 4096 x 50257 x 2048, where an end comes after every 32 stages, 625 to 650 us by the card (67 %) and its gradient to E5M2 737 to 764 (54 %), the product to bf16 680.
#pragma once

#include "gemm_op.hpp"

namespace fp8mm {

struct LossArgs : OpArgs {
    const int64_t* labels;                      // M; negative: no label
    const float* lse;                           // M (the gradient)
    const float* dloss;                         // one or M (the gradient)
    void* partials;                             // M pairs for each block of columns; behind the most that there can be: the labels' logits
    int64_t first;                              // the label that the first column stands for
    float z_weight;
    int dloss_per_row;
    int wide_cols;                              // tiled kernel, both widths in one launch: tile columns 256 wide
};

struct LossPair { float ref, sum; };
__host__ __device__ inline int64_t loss_blocks_most(int64_t N) { return N / 32 + (N % 32 != 0); }
__host__ __device__ inline float* loss_targets(const LossArgs& o, int64_t M, int64_t N) { return (float*)((LossPair*)o.partials + M * loss_blocks_most(N)); }

// The products of gemm_op.hpp with these ends; loss, lse: of OP_LOSS.
int launch_gemm_loss(const GemmArgs& g, const LossArgs& o, float* loss, float* lse);

// Tiles of 256 rows (gemm_op_tiled.hip): A stored M x K, both operands in E4M3; small tiles (gemm_op_small.hip): other formats than E4M3 on
// 64 x 64 and the fp16 instructions.
int launch_loss_tiled_l0_a0(const GemmArgs& g, const LossArgs& o);
int launch_loss_tiled_l0_a1(const GemmArgs& g, const LossArgs& o);
int launch_loss_tiled_l1_a0(const GemmArgs& g, const LossArgs& o);
int launch_loss_tiled_l1_a1(const GemmArgs& g, const LossArgs& o);
// The kernel for any shape (gemm_mfma_any.hip), both operands in E4M3; width: 256 or 128 columns a tile.
int launch_loss_any_l0(const GemmArgs& g, const LossArgs& o, int width);
int launch_loss_any_l1(const GemmArgs& g, const LossArgs& o, int width);
int launch_loss_any_l2(const GemmArgs& g, const LossArgs& o, int width);
int launch_loss_any_l3(const GemmArgs& g, const LossArgs& o, int width);
int launch_loss_small_l0(const GemmArgs& g, const LossArgs& o, int form);
int launch_loss_small_l1(const GemmArgs& g, const LossArgs& o, int form);
int launch_loss_small_l2(const GemmArgs& g, const LossArgs& o, int form);
int launch_loss_small_l3(const GemmArgs& g, const LossArgs& o, int form);

// The arguments that a kernel of the operator takes.
template <bool LOSS> struct ArgsOf { typedef OpArgs type; };
template <> struct ArgsOf<true> { typedef LossArgs type; };

namespace {

constexpr float kLog2e = 1.44269504088896340736f;

// The pair of a row of which a lane holds C values x, t = g x (g > 0; outside: -infinity), and LANES lanes, FIRST apart, the rest; in all of these lanes.
template <int C, int LANES, int FIRST = 1>
__device__ __forceinline__ LossPair loss_pair(const float (&x)[C], float g = 1.0f)
{
    float top = x[0];
#pragma unroll
    for (int i = 1; i < C; ++i) top = __builtin_fmaxf(top, x[i]);
    top *= g;
#pragma unroll
    for (int d = FIRST; d < LANES * FIRST; d <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, d, 64));
    constexpr float most = 3.4028234663852886e38f;
    const float ref = __builtin_fminf(__builtin_fmaxf(top, -most), most);
    // (four runs: fewer roundings behind one another)
    float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < C; ++i) part[i % 4] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], g, -ref));
    float s = (part[0] + part[1]) + (part[2] + part[3]);
#pragma unroll
    for (int d = FIRST; d < LANES * FIRST; d <<= 1) s += __shfl_xor(s, d, 64);
    return {ref, s};
}

// The column of a row's label (outside [0, N): in another piece), -1 of a row without one.
__device__ __forceinline__ int64_t column_of_label(const LossArgs& o, int64_t y) { return y < 0 ? -1 : y < o.first ? -2 : y - o.first; }
__device__ __forceinline__ int64_t label_column(const LossArgs& o, int64_t row)
{
    return column_of_label(o, o.labels[row]);
}

// A row's part in its gradient.
struct LossRow { float lse2, scale, dloss; int64_t label; };     // lse log2(e); dloss (1 + 2 w lse); as above

__device__ __forceinline__ LossRow loss_row(const LossArgs& o, float lse, float dloss, int64_t label)
{
    return {lse * kLog2e, o.z_weight != 0.0f ? dloss * __builtin_fmaf(2.0f * o.z_weight, lse, 1.0f) : dloss, dloss, column_of_label(o, label)};
}
__device__ __forceinline__ LossRow loss_row(const LossArgs& o, int64_t row) { return loss_row(o, o.lse[row], o.dloss[o.dloss_per_row ? row : 0], o.labels[row]); }

// x: t - lse2 of G rows of W columns -> the gradient, stored; scale, dloss, label: of the rows (label as above, of any integer type).  Returns the largest magnitude.
template <int G, int W, class I>
__device__ __forceinline__ unsigned loss_grad_finish(const LossArgs& o, void* D, int64_t N, const OutRows<G>& t, float (&x)[G * W], const float (&scale)[G], const float (&dloss)[G],
                                                     const I (&label)[G], float sD)
{
    bool some = false;
#pragma unroll
    for (int g = 0; g < G; ++g) {
#pragma unroll
        for (int i = 0; i < W; ++i) x[g * W + i] = __builtin_amdgcn_exp2f(x[g * W + i]) * scale[g];
        some |= label[g] == (I)-1 || (label[g] >= (I)t.col && label[g] < (I)(t.col + W));
    }
    // rows without a label (whatever their logits) and the labels' own columns: in few of a tile's steps
    if (__any(some)) {
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float y = x[g * W + i];
                x[g * W + i] = label[g] == (I)-1 ? 0.0f : label[g] == (I)(t.col + i) ? y - dloss[g] : y;
            }
    }
    zero_outside<G, W>(t, x);
    const unsigned top = max_bits_of<G * W>(x);
    store_rows<G, W>(D, o.out_kind, rows_at(t, N, 0), x, sD, top);
    return top;
}

// One row of W columns, `left` (>= 1) of them inside, z: the logits.
template <int W>
__device__ __forceinline__ unsigned loss_grad_row(const LossArgs& o, void* D, int64_t N, int64_t row, int64_t col, int left, const float (&z)[W], float sD)
{
    const LossRow r = loss_row(o, row);
    const OutRows<1> t = {{row}, col, left, 1u, false};
    float x[W];
#pragma unroll
    for (int i = 0; i < W; ++i) x[i] = __builtin_fmaf(z[i], kLog2e, -r.lse2);
    const float scale[1] = {r.scale}, dloss[1] = {r.dloss};
    const int64_t label[1] = {r.label};
    return loss_grad_finish<1, W>(o, D, N, t, x, scale, dloss, label, sD);
}

// The forward pass, W columns of a row, `left` (may be <= 0) of them inside: the label's logit is left in memory, z becomes t.
template <int W>
__device__ __forceinline__ void loss_logits(const LossArgs& o, int64_t M, int64_t N, int64_t row, int64_t col, int left, int64_t label, float (&z)[W])
{
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if (row < M && i < left && label == col + i) loss_targets(o, M, N)[row] = z[i];
        z[i] = i < left ? z[i] * kLog2e : -__builtin_inff();
    }
}

}  // namespace
}  // namespace fp8mm
