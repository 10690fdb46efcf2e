// What the products with an operator behind them share (fp8_gemm_act, fp8_gemm_act_grad, fp8_gemm_gated,
// fp8_gemm_gated_grad; gfx950): the arguments, the activations, and the step from sums to outputs, a few neighbouring
// columns of a row at a time, which every kernel form ends with.
//
//   c = acc / (sA_i sB_j), in 32 bits from the 32-bit sums (arXiv 2209.05433, Section 2: factors taken out once per dot product)
//   OP_ACT         z = c + bias_j, y = act(z) + residual;  z may be kept
//   OP_ACT_GRAD    y = c act'(z), z as kept;  column sums of y
//   OP_GATED       g and u are the columns j and N + j of a product 2 N wide;  y = act(g) u;  g and u may be kept
//   OP_GATED_GRAD  y = (c u act'(g), c act(g)) to the columns j and N + j of an output 2 N wide
//   amax = max |y|;  D = cast_out(y), or encode(y sD) for FP8 outputs
//
// Everything between the sums and the output is in 32 bits and rounded once, at a store.
#pragma once

#include "gemm_common.hpp"

#include <atomic>

namespace fp8mm {

enum { OP_ACT = 0, OP_ACT_GRAD = 1, OP_GATED = 2, OP_GATED_GRAD = 3 };
// Factors of B: one; one of the gate's and one of the other projection's columns; one per column (2 N of them for OP_GATED).
enum { B_ONE = 0, B_PAIR = 1, B_COLUMN = 2 };

struct OpArgs : EpilogueArgs {                  // (sA_dev, sB_dev: given; b_per_col: not looked at)
    float* sums;                                // null or partial column sums, a row of N for each kOpSumRows rows at least
    const void* bias;                           // null or N values
    const void* side;                           // residual (M x N or null), z (M x N), or g | u (M x 2 N)
    void* kept;                                 // null, z (M x N) or g | u (M x 2 N)
    int op, act;
    int bias_dtype, side_dtype, kept_dtype;     // fp8_dtype_t
    int b_factors;                              // B_*
};

constexpr int kOpSumRows = 32;                  // rows of the output behind one row of partial column sums, at least
inline bool op_pair_in(int op) { return op == OP_GATED; }             // B has two columns for each output column
inline int64_t op_width(int op, int64_t N) { return op == OP_GATED_GRAD ? 2 * N : N; }

// g: operands, D, M, N (columns of D, or of either half), K; g.ep is not looked at.
int launch_gemm_op(const GemmArgs& g, const OpArgs& o, float* dbias);

// The kernel of small tiles (gemm_op_small.hip), one translation unit per pair of storage orders; form: SMALL_*, of the 64 x 64 ones
// those of chunks of 128 where both operands are contiguous along K.  g.N >= 16 where op(B)'s column pairs are contiguous along N.
#define FP8MM_OP_SMALL_NAME_(l) launch_op_small_l##l
#define FP8MM_OP_SMALL_NAME(l) FP8MM_OP_SMALL_NAME_(l)
int FP8MM_OP_SMALL_NAME(0)(const GemmArgs& g, const OpArgs& o, int form);
int FP8MM_OP_SMALL_NAME(1)(const GemmArgs& g, const OpArgs& o, int form);
int FP8MM_OP_SMALL_NAME(2)(const GemmArgs& g, const OpArgs& o, int form);
int FP8MM_OP_SMALL_NAME(3)(const GemmArgs& g, const OpArgs& o, int form);

// The tiled kernel (gemm_op_tiled.hip), one translation unit per (storage orders, accumulation mode); g.tile_n: 256 or 128 columns of
// op(B).  The conditions of the plain product's tiled kernel, and for the gated block a second projection that begins on a 16-byte boundary less
// than 2^32 bytes behind the first.
#define FP8MM_OP_TILED_NAME_(l, a) launch_op_tiled_l##l##_a##a
#define FP8MM_OP_TILED_NAME(l, a) FP8MM_OP_TILED_NAME_(l, a)
#define FP8MM_DECLARE_OP_TILED(l) \
    int FP8MM_OP_TILED_NAME(l, 0)(const GemmArgs& g, const OpArgs& o); \
    int FP8MM_OP_TILED_NAME(l, 1)(const GemmArgs& g, const OpArgs& o);
FP8MM_DECLARE_OP_TILED(0)
FP8MM_DECLARE_OP_TILED(1)
FP8MM_DECLARE_OP_TILED(2)
FP8MM_DECLARE_OP_TILED(3)
#undef FP8MM_DECLARE_OP_TILED

// Raises a kernel's limit of dynamic LDS, once per device (`done`: of this kernel).
int raise_lds_limit(const void* kernel, int bytes, std::atomic<unsigned long long>& done);

namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));
typedef __bf16 op_bf16x2 __attribute__((ext_vector_type(2)));
typedef float op_f32x2 __attribute__((ext_vector_type(2)));

// ---- activations ------------------------------------------------------------------------------------------------
// With s(t) = 1 / (1 + e^-t): SiLU z s(z); GELU z Phi(z); its tanh form z s(2 k (z + 0.044715 z^3)), k = sqrt(2 / pi), since
// (1 + tanh t) / 2 = s(2 t).  Beyond |z| = 16 the tails are 0 and 1 in 32 bits; the polynomial and the products of the derivative are
// taken of the clamped z (NaN passes), so that nothing there becomes inf x 0.  act(-inf) is the limit, 0; NaN stays NaN.
// The exponential and the reciprocal are the instructions (1 ulp each).
__device__ __forceinline__ float op_clamp(float z, float most) { return z > most ? most : z < -most ? -most : z; }
__device__ __forceinline__ float op_sigmoid(float t) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * t)); }

template <int ACT>
__device__ __forceinline__ void act_both(float z, float& value, float& slope)
{
    if (ACT == FP8_ACT_NONE) {
        value = z; slope = 1.0f;
    } else if (ACT == FP8_ACT_RELU) {
        value = z < 0.0f ? 0.0f : z;
        slope = z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z;
    } else if (ACT == FP8_ACT_SILU) {
        const float zc = op_clamp(z, 128.0f), s = op_sigmoid(zc);
        value = (z < -128.0f ? -128.0f : z) * s;
        slope = s * (1.0f + zc * (1.0f - s));
    } else if (ACT == FP8_ACT_GELU) {
        const float zc = op_clamp(z, 16.0f), p = 0.5f + 0.5f * erff(0.70710678f * zc);
        value = (z < -16.0f ? -16.0f : z) * p;
        slope = p + zc * (0.39894228f * __builtin_amdgcn_exp2f(-0.72134752f * zc * zc));
    } else {
        const float zc = op_clamp(z, 16.0f), q = zc * zc;
        const float s = op_sigmoid(1.59576912f * zc * (1.0f + 0.044715f * q));
        value = (z < -16.0f ? -16.0f : z) * s;
        slope = s + zc * s * (1.0f - s) * 1.59576912f * (1.0f + 0.134145f * q);
    }
}

template <int W, int ACT>
__device__ __forceinline__ void act_each(const float (&z)[W], float (&value)[W], float (&slope)[W])
{
#pragma unroll
    for (int i = 0; i < W; ++i) act_both<ACT>(z[i], value[i], slope[i]);
}

template <int W>
__device__ __forceinline__ void act_row(int act, const float (&z)[W], float (&value)[W], float (&slope)[W])
{
    switch (act) {
        case FP8_ACT_NONE: act_each<W, FP8_ACT_NONE>(z, value, slope); break;
        case FP8_ACT_RELU: act_each<W, FP8_ACT_RELU>(z, value, slope); break;
        case FP8_ACT_GELU: act_each<W, FP8_ACT_GELU>(z, value, slope); break;
        case FP8_ACT_SILU: act_each<W, FP8_ACT_SILU>(z, value, slope); break;
        default: act_each<W, FP8_ACT_GELU_TANH>(z, value, slope); break;
    }
}

// ---- W neighbouring values of a row in memory, `left` of them there (the rest: zeros) ----------------------------------
template <int W>
__device__ __forceinline__ void load_row(const void* p, int dtype, int64_t at, int left, float (&v)[W])
{
    static_assert(W == 4 || W == 8, "two sizes of pieces");
    if (dtype == FP8_F32) {
        const float* f = (const float*)p + at;
        if (left >= W) {
#pragma unroll
            for (int i = 0; i < W / 4; ++i) {
                const u32x4 x = *(const u32x4_any*)(f + 4 * i);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[4 * i + j] = as_f32(x[j]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] = i < left ? f[i] : 0.0f;
        }
        return;
    }
    const unsigned short* h = (const unsigned short*)p + at;
    if (left >= W) {
        unsigned x[W / 2];
        if (W == 8) {
            const u32x4 t = *(const u32x4_any*)h;
#pragma unroll
            for (int j = 0; j < W / 2; ++j) x[j] = t[j & 3];
        } else {
            const u32x2 t = *(const u32x2_any*)h;
#pragma unroll
            for (int j = 0; j < W / 2; ++j) x[j] = t[j & 1];
        }
#pragma unroll
        for (int j = 0; j < W / 2; ++j) { v[2 * j] = as_f32(x[j] << 16); v[2 * j + 1] = as_f32(x[j] & 0xffff0000u); }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = i < left ? as_f32((unsigned)h[i] << 16) : 0.0f;
    }
}

// out_kind: as of the product's output (the first two are fp8_dtype_t); sD: of FP8 kinds.  quad_max: the largest magnitude of v as bits.
template <int W>
__device__ __forceinline__ void store_row(void* p, int out_kind, int64_t at, int left, const float (&v)[W], float sD, unsigned max_bits)
{
    if (out_kind == OUT_F32) {
        float* f = (float*)p + at;
        if (left >= W) {
#pragma unroll
            for (int i = 0; i < W / 4; ++i)
                *(u32x4_any*)(f + 4 * i) = (u32x4){as_u32(v[4 * i]), as_u32(v[4 * i + 1]), as_u32(v[4 * i + 2]), as_u32(v[4 * i + 3])};
        } else {
#pragma unroll
            for (int i = 0; i < W - 1; ++i) if (i < left) f[i] = v[i];
        }
    } else if (out_kind == OUT_BF16) {
        unsigned short* h = (unsigned short*)p + at;
        unsigned x[W / 2];
#pragma unroll
        for (int j = 0; j < W / 2; ++j) x[j] = __builtin_bit_cast(unsigned, __builtin_convertvector((op_f32x2){v[2 * j], v[2 * j + 1]}, op_bf16x2));
        if (left >= W) {
            if (W == 8) *(u32x4_any*)h = (u32x4){x[0], x[1], x[W / 2 - 2], x[W / 2 - 1]};
            else *(u32x2_any*)h = (u32x2){x[0], x[1]};
        } else {
#pragma unroll
            for (int i = 0; i < W - 1; ++i) if (i < left) h[i] = (unsigned short)(x[i >> 1] >> (16 * (i & 1)));
        }
    } else {
        // (the largest product tells whether anything has to be clamped or looked at one by one)
        const bool e4m3 = out_kind == OUT_E4M3, inside = __builtin_fabsf(as_f32(max_bits) * sD) <= (e4m3 ? 448.0f : 57344.0f);
        unsigned x[W / 4];
#pragma unroll
        for (int j = 0; j < W / 4; ++j) {
            const float a = v[4 * j] * sD, b = v[4 * j + 1] * sD, c = v[4 * j + 2] * sD, d = v[4 * j + 3] * sD;
            x[j] = inside ? (e4m3 ? encode4_inside<FP8_E4M3>(a, b, c, d) : encode4_inside<FP8_E5M2>(a, b, c, d))
                          : (e4m3 ? encode4<FP8_E4M3>(a, b, c, d) : encode4<FP8_E5M2>(a, b, c, d));
        }
        uint8_t* q = (uint8_t*)p + at;
        if (left >= W) {
            if (W == 8) *(u32x2_any*)q = (u32x2){x[0], x[W / 4 - 1]};
            else *(unsigned __attribute__((aligned(1)))*)q = x[0];
        } else {
#pragma unroll
            for (int i = 0; i < W - 1; ++i) if (i < left) q[i] = (uint8_t)(x[i >> 2] >> (8 * (i & 3)));
        }
    }
}

// NaN patterns sort above infinity.
template <int W>
__device__ __forceinline__ unsigned max_bits_of(const float (&v)[W], int left)
{
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) m = max(m, i < left ? as_u32(v[i]) & 0x7fffffffu : 0u);
    return m;
}

// ---- sums -> outputs ---------------------------------------------------------------------------------------------------
// W columns from `col` on of row `row`, `left` (>= 1) of them inside; y, u: the values of c (u: of the second projection).  y is left as
// what goes into the column sums (zeros outside).  Returns the largest |output| as bits.
template <int W, bool PAIR>
__device__ __forceinline__ unsigned op_row(const OpArgs& o, void* D, int64_t N, int64_t row, int64_t col, int left, float (&y)[W], const float (&u)[W],
                                           const float (&bias)[W], float sD)
{
    float value[W], slope[W], side[W];
    if (PAIR) {                                                           // OP_GATED
        if (o.kept) {
            store_row<W>(o.kept, o.kept_dtype, row * 2 * N + col, left, y, 1.0f, 0);
            store_row<W>(o.kept, o.kept_dtype, row * 2 * N + N + col, left, u, 1.0f, 0);
        }
        act_row<W>(o.act, y, value, slope);
#pragma unroll
        for (int i = 0; i < W; ++i) value[i] *= u[i];
        const unsigned top = max_bits_of<W>(value, left);
        store_row<W>(D, o.out_kind, row * N + col, left, value, sD, top);
        return top;
    }
    if (o.op == OP_ACT) {
#pragma unroll
        for (int i = 0; i < W; ++i) y[i] += bias[i];
        if (o.kept) store_row<W>(o.kept, o.kept_dtype, row * N + col, left, y, 1.0f, 0);
        act_row<W>(o.act, y, value, slope);
        if (o.side) {
            load_row<W>(o.side, o.side_dtype, row * N + col, left, side);
#pragma unroll
            for (int i = 0; i < W; ++i) value[i] += side[i];
        }
        const unsigned top = max_bits_of<W>(value, left);
        store_row<W>(D, o.out_kind, row * N + col, left, value, sD, top);
        return top;
    }
    const int64_t width = o.op == OP_GATED_GRAD ? 2 * N : N;
    load_row<W>(o.side, o.side_dtype, row * width + col, left, side);
    act_row<W>(o.act, side, value, slope);
    unsigned top = 0;
    if (o.op == OP_GATED_GRAD) {
        load_row<W>(o.side, o.side_dtype, row * width + N + col, left, side);
#pragma unroll
        for (int i = 0; i < W; ++i) { value[i] *= y[i]; slope[i] *= side[i]; }
        top = max_bits_of<W>(value, left);
        store_row<W>(D, o.out_kind, row * width + N + col, left, value, sD, top);
    }
#pragma unroll
    for (int i = 0; i < W; ++i) y[i] = i < left ? y[i] * slope[i] : 0.0f;
    const unsigned top_y = max_bits_of<W>(y, left);
    store_row<W>(D, o.out_kind, row * width + col, left, y, sD, top_y);
    return max(top, top_y);
}

// 1 / the factor of a column of the product (up: of the second projection), in 64 bits: with 1 / sA it is rounded once.
__device__ __forceinline__ double op_column_factor(const OpArgs& o, int64_t N, int64_t col, bool up)
{
    return 1.0 / (double)o.sB_dev[o.b_factors == B_COLUMN ? col + (up ? N : 0) : o.b_factors == B_PAIR && up ? 1 : 0];
}

}  // namespace
}  // namespace fp8mm
