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
    unsigned* tops;                             // null or the workgroups' maxima, which then do not go to amax_out
    const void* bias;                           // null or N values
    const void* side;                           // residual (M x N or null), z (M x N), or g | u (M x 2 N)
    void* kept;                                 // null, z (M x N) or g | u (M x 2 N)
    int op, act;
    int bias_dtype, side_dtype, kept_dtype;     // fp8_dtype_t
    int b_factors;                              // B_*
};

constexpr int kOpSumRows = 32;                  // rows of the output behind one row of partial column sums, at least
inline bool op_pair_in(int op) { return op == OP_GATED; }             // B has two columns for each output column

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
// op(B); g.wide_cols > 0: that many tile columns of 256 and narrow ones for the rest.  The conditions of the plain product's tiled kernel; B in E4M3 (as weights and activations are); for the gated block a second projection
// that begins on a 16-byte boundary less than 2^32 bytes behind the first.
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

// The kernel of up to 16 rows (gemm_op_skinny.hip): A stored M x K, B stored N x K, rows on 16-byte boundaries, where it pays.
bool op_skinny_takes(const GemmArgs& g, bool pair);
int launch_op_skinny(const GemmArgs& g, const OpArgs& o);

// Raises a kernel's limit of dynamic LDS, once per device (`done`: of this kernel).
int raise_lds_limit(const void* kernel, int bytes, std::atomic<unsigned long long>& done);

namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));
typedef __bf16 op_bf16x2 __attribute__((ext_vector_type(2)));
typedef float op_f32x2 __attribute__((ext_vector_type(2)));

// ---- activations ------------------------------------------------------------------------------------------------
// With s(t) = 1 / (1 + e^-t): SiLU z s(z); GELU z Phi(z); its tanh form z s(2 k (z + 0.044715 z^3)), k = sqrt(2 / pi), since
// (1 + tanh t) / 2 = s(2 t).  The exponential and the reciprocal are the instructions (1 ulp each), four slots of the vector ALU each.
// Phi, where the value alone is asked for: s(z P(z^2)), P fitted to log(Phi(z) / Phi(-z)) / z with degree 6, Phi within 3.7e-8 over the
// whole range (beyond the fit z P only grows) but for rounding: 19 slots.  With the derivative, whose density needs e^(-z^2 / 2) anyway, Hastings' rational
// approximation of the error function (Abramowitz and Stegun 7.1.26): with x = |z| / sqrt(2), t = 1 / (1 + 0.3275911 x)
// 1 - Phi(|z|) = t (a1 + t (a2 + ...)) e^(-x^2) / 2 within 7.5e-8 but for rounding: 24 slots for the derivative.  (The library's erff: about 100, and 4096 x 6144
// outputs spent 15 us a round in it.)
// Measured at 4 million z between -20 and 31, |error| / |z| of the value at most 1.7e-7 (GELU), 1.5e-7 (its tanh form, SiLU), GELU's beside its
// derivative 3.0e-7; of the derivative 3.1e-7 (GELU), 2.0e-6 (tanh form), 9.8e-7 (SiLU).  GELU's bounds are absolute: of its left tail little
// is right beyond z = -5 (a value of 1e-6), by 1.4e-5 of the value at -3, 1 % at -5, 94 % at -6, as of (1 + erf) / 2 in 32 bits, where 1 + erf cancels.
// The other two keep their digits there.
// Beyond |z| = 16 (SiLU: 128) the tails are 0 and 1 in 32 bits; where z would come in as inf x 0 it is held there (a NaN comes through the other
// factor): act(-inf) is the limit, 0.
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
        const float s = op_sigmoid(z);
        value = __builtin_amdgcn_fmed3f(z, -128.0f, __builtin_inff()) * s;
        slope = s * __builtin_fmaf(__builtin_amdgcn_fmed3f(z, -128.0f, 128.0f), 1.0f - s, 1.0f);
    } else if (ACT == FP8_ACT_GELU) {
        const float e = __builtin_amdgcn_exp2f(-0.72134752f * z * z);                         // e^(-z^2 / 2)
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.23164191f, __builtin_fabsf(z), 1.0f));
        float q = __builtin_fmaf(0.530702714f, t, -0.726576013f);                               // (the halves of a5 .. a1)
        q = __builtin_fmaf(q, t, 0.710706870f);
        q = __builtin_fmaf(q, t, -0.142248368f);
        q = __builtin_fmaf(q, t, 0.127414796f) * t * e;
        const float p = z < 0.0f ? q : 1.0f - q;
        value = __builtin_amdgcn_fmed3f(z, -16.0f, __builtin_inff()) * p;
        slope = __builtin_fmaf(__builtin_amdgcn_fmed3f(z, -16.0f, 16.0f) * 0.39894228f, e, p);
    } else {
        const float zc = __builtin_amdgcn_fmed3f(z, -16.0f, 16.0f), q = z == z ? zc * zc : z;
        const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(zc * __builtin_fmaf(-0.10294324f, q, -2.3022082f)));
        value = __builtin_amdgcn_fmed3f(z, -16.0f, __builtin_inff()) * s;
        slope = __builtin_fmaf(zc * s * (1.0f - s) * 1.59576912f, __builtin_fmaf(0.134145f, q, 1.0f), s);
    }
}

// Both GELUs where nobody asks for the derivative; coefficients of -P / log(2), and of -2 k (1 + 0.044715 q) / log(2).
__device__ __forceinline__ float gelu_value(float z)
{
    const float q = z * z;
    float p = __builtin_fmaf(-5.06754327e-09f, q, 3.81639751e-07f);
    p = __builtin_fmaf(p, q, -1.14399163e-05f);
    p = __builtin_fmaf(p, q, 0.00015958029f);
    p = __builtin_fmaf(p, q, 9.40485625e-05f);
    p = __builtin_fmaf(p, q, -0.104835123f);
    p = __builtin_fmaf(p, q, -2.30220938f);
    return __builtin_amdgcn_fmed3f(z, -16.0f, __builtin_inff()) * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * p));
}
__device__ __forceinline__ float gelu_tanh_value(float z)
{
    const float p = __builtin_fmaf(-0.10294324f, z * z, -2.3022082f);
    return __builtin_amdgcn_fmed3f(z, -16.0f, __builtin_inff()) * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * p));
}

template <int E, int ACT, bool VALUE_ONLY>
__device__ __forceinline__ void act_each(const float (&z)[E], float (&value)[E], float (&slope)[E])
{
#pragma unroll
    for (int i = 0; i < E; ++i) {
        if (ACT == FP8_ACT_GELU && VALUE_ONLY) value[i] = gelu_value(z[i]);
        else if (ACT == FP8_ACT_GELU_TANH && VALUE_ONLY) value[i] = gelu_tanh_value(z[i]);
        else act_both<ACT>(z[i], value[i], slope[i]);
    }
}

// VALUE_ONLY: slope is not looked at.
template <int E, bool VALUE_ONLY>
__device__ __forceinline__ void act_all(int act, const float (&z)[E], float (&value)[E], float (&slope)[E])
{
    switch (act) {
        case FP8_ACT_NONE: act_each<E, FP8_ACT_NONE, VALUE_ONLY>(z, value, slope); break;
        case FP8_ACT_RELU: act_each<E, FP8_ACT_RELU, VALUE_ONLY>(z, value, slope); break;
        case FP8_ACT_GELU: act_each<E, FP8_ACT_GELU, VALUE_ONLY>(z, value, slope); break;
        case FP8_ACT_SILU: act_each<E, FP8_ACT_SILU, VALUE_ONLY>(z, value, slope); break;
        default: act_each<E, FP8_ACT_GELU_TANH, VALUE_ONLY>(z, value, slope); break;
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

// Where G rows of W values go: the index of each row's first value, how many of the W columns are inside, which of the rows (whole: all rows
// and columns, the same for the wave).
template <int G> struct RowsAt { int64_t at[G]; int left; unsigned rows; bool whole; };

template <int G, int W, class F>
__device__ __forceinline__ void each_row(const RowsAt<G>& t, F store)
{
    if (t.whole) {
#pragma unroll
        for (int g = 0; g < G; ++g) store(g);
    } else {
#pragma unroll
        for (int g = 0; g < G; ++g) if (t.rows >> g & 1) store(g);
    }
}

// A lane's columns of a row.  At a tile's end (several rows at a time) the waves write whole lines, which push no operands out of the caches: 4096 x 6144
// x 2048 114.7 -> 113.2 us, 8192 x 6144 gradients of a gated block 229.4 -> 227.1, 1537 x 5504 67.0 -> 65.2; with the product that reads the output behind
// them 203 -> 200 and 289.5 -> 288.5, the gated block of 8192 rows 494 -> 484, of 300 rows 53.8 -> 54.0.
template <int G, class V> __device__ __forceinline__ void store_columns(void* p, V v)
{
    typedef V any __attribute__((aligned(1)));
    if (G > 1) __builtin_nontemporal_store(v, (any*)p);
    else *(any*)p = v;
}

// out_kind: as of a product's output (the first two are fp8_dtype_t); sD: of FP8 kinds, max_bits: the largest magnitude of v there, as bits.
template <int G, int W>
__device__ __forceinline__ void store_rows(void* p, int out_kind, const RowsAt<G>& t, const float (&v)[G * W], float sD, unsigned max_bits)
{
    if (out_kind == OUT_BF16) {
        unsigned x[G * W / 2];
#pragma unroll
        for (int j = 0; j < G * W / 2; ++j) x[j] = __builtin_bit_cast(unsigned, __builtin_convertvector((op_f32x2){v[2 * j], v[2 * j + 1]}, op_bf16x2));
        each_row<G, W>(t, [&](int g) __attribute__((always_inline)) {
            unsigned short* h = (unsigned short*)p + t.at[g];
            const unsigned* r = x + g * (W / 2);
            if (t.whole || t.left >= W) {
                if (W == 8) store_columns<G>(h, (u32x4){r[0], r[1], r[W / 2 - 2], r[W / 2 - 1]});
                else store_columns<G>(h, (u32x2){r[0], r[1]});
            } else {
#pragma unroll
                for (int i = 0; i < W - 1; ++i) if (i < t.left) h[i] = (unsigned short)(r[i >> 1] >> (16 * (i & 1)));
            }
        });
    } else if (out_kind == OUT_F32) {
        each_row<G, W>(t, [&](int g) __attribute__((always_inline)) {
            float* f = (float*)p + t.at[g];
            const float* r = v + g * W;
            if (t.whole || t.left >= W) {
#pragma unroll
                for (int i = 0; i < W / 4; ++i)
                    store_columns<G>(f + 4 * i, (u32x4){as_u32(r[4 * i]), as_u32(r[4 * i + 1]), as_u32(r[4 * i + 2]), as_u32(r[4 * i + 3])});
            } else {
#pragma unroll
                for (int i = 0; i < W - 1; ++i) if (i < t.left) f[i] = r[i];
            }
        });
    } else {
        // (the largest product tells whether anything has to be clamped, or looked at one by one: not where all are finite.  With a factor from past maxima
        // one of a step's thousand values lies outside the format at nearly every step)
        const float largest = __builtin_fabsf(as_f32(max_bits) * sD);
        const bool e4m3 = out_kind == OUT_E4M3, inside = largest <= (e4m3 ? 448.0f : 57344.0f), finite = largest < __builtin_inff();
        unsigned x[G * W / 4];
        float y[G * W];
#pragma unroll
        for (int j = 0; j < G * W; ++j) y[j] = v[j] * sD;
        if (__all(inside)) {
            if (e4m3) {
#pragma unroll
                for (int j = 0; j < G * W / 4; ++j) x[j] = encode4_inside<FP8_E4M3>(y[4 * j], y[4 * j + 1], y[4 * j + 2], y[4 * j + 3]);
            } else {
#pragma unroll
                for (int j = 0; j < G * W / 4; ++j) x[j] = encode4_inside<FP8_E5M2>(y[4 * j], y[4 * j + 1], y[4 * j + 2], y[4 * j + 3]);
            }
        } else if (__all(finite)) {
            if (e4m3) {
#pragma unroll
                for (int j = 0; j < G * W / 4; ++j) x[j] = cvt_pair<FP8_E4M3, true>(y[4 * j + 2], y[4 * j + 3], cvt_pair<FP8_E4M3, false>(y[4 * j], y[4 * j + 1], 0u));
            } else {
#pragma unroll
                for (int j = 0; j < G * W / 4; ++j) x[j] = cvt_pair<FP8_E5M2, true>(y[4 * j + 2], y[4 * j + 3], cvt_pair<FP8_E5M2, false>(y[4 * j], y[4 * j + 1], 0u));
            }
        } else {
#pragma unroll
            for (int j = 0; j < G * W / 4; ++j)
                x[j] = e4m3 ? encode4_bits<FP8_E4M3>(y[4 * j], y[4 * j + 1], y[4 * j + 2], y[4 * j + 3]) : encode4_bits<FP8_E5M2>(y[4 * j], y[4 * j + 1], y[4 * j + 2], y[4 * j + 3]);
        }
        each_row<G, W>(t, [&](int g) __attribute__((always_inline)) {
            uint8_t* q = (uint8_t*)p + t.at[g];
            const unsigned* r = x + g * (W / 4);
            if (t.whole || t.left >= W) {
                if (W == 8) store_columns<G>(q, (u32x2){r[0], r[W / 4 - 1]});
                else store_columns<G>(q, r[0]);
            } else {
#pragma unroll
                for (int i = 0; i < W - 1; ++i) if (i < t.left) q[i] = (uint8_t)(r[i >> 2] >> (8 * (i & 3)));
            }
        });
    }
}

// ---- sums -> outputs ---------------------------------------------------------------------------------------------------
// Which G rows of an output a lane finishes: W columns from `col` on, `left` of them inside (>= 1 for a lane with rows).
template <int G> struct OutRows { int64_t row[G]; int64_t col; int left; unsigned rows; bool whole; };

template <int G>
__device__ __forceinline__ RowsAt<G> rows_at(const OutRows<G>& t, int64_t width, int64_t more)
{
    RowsAt<G> r;
#pragma unroll
    for (int g = 0; g < G; ++g) r.at[g] = t.row[g] * width + t.col + more;
    r.left = t.left; r.rows = t.rows; r.whole = t.whole;
    return r;
}

// Zeros in the place of what lies outside.
template <int G, int W>
__device__ __forceinline__ void zero_outside(const OutRows<G>& t, float (&v)[G * W])
{
    if (t.whole) return;
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int i = 0; i < W; ++i) v[g * W + i] = (t.rows >> g & 1) && i < t.left ? v[g * W + i] : 0.0f;
}

// The largest magnitude as bits (a NaN stays one: its pattern sorts above infinity).
template <int E>
__device__ __forceinline__ unsigned max_bits_of(const float (&v)[E])
{
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < E; ++i) m = __builtin_elementwise_maximum(m, __builtin_fabsf(v[i]));     // (two values an instruction)
    return as_u32(m) & 0x7fffffffu;
}

// y, u: the values of c (u: of the second projection); a, b: what o.side has there (b: of the second projection; OP_ACT: a is zero
// without a residual).  OP_ACT_GRAD leaves in y what goes into the column sums (zeros outside).  Returns the largest |output| as bits.
// Several rows at a time, so that the branches on the call's kinds are taken once for all of them: with one wave a SIMD
// nothing hides a branch either (8 values a time: 945 cycles of a 256-wide tile's end were 60 instructions and 15 branches).
template <int G, int W, int OP>
__device__ __forceinline__ unsigned op_finish(const OpArgs& o, void* D, int64_t N, const OutRows<G>& t, float (&y)[G * W], float (&u)[G * W], const float (&bias)[W],
                                              const float (&a)[G * W], const float (&b)[G * W], float sD)
{
    constexpr int E = G * W;
    float value[E], slope[E];
    unsigned top = 0;
    if (OP == OP_ACT || OP == OP_GATED) {
        if (OP == OP_ACT) {
#pragma unroll
            for (int i = 0; i < E; ++i) y[i] += bias[i % W];
        }
        if (o.kept) {
            store_rows<G, W>(o.kept, o.kept_dtype, rows_at(t, OP == OP_GATED ? 2 * N : N, 0), y, 1.0f, 0);
            if (OP == OP_GATED) store_rows<G, W>(o.kept, o.kept_dtype, rows_at(t, 2 * N, N), u, 1.0f, 0);
        }
        act_all<E, true>(o.act, y, value, slope);
#pragma unroll
        for (int i = 0; i < E; ++i) value[i] = OP == OP_GATED ? value[i] * u[i] : value[i] + a[i];
        zero_outside<G, W>(t, value);
        top = max_bits_of<E>(value);
        store_rows<G, W>(D, o.out_kind, rows_at(t, N, 0), value, sD, top);
        return top;
    }
    act_all<E, false>(o.act, a, value, slope);
    const int64_t width = OP == OP_GATED_GRAD ? 2 * N : N;
    unsigned top_u = 0;
    if (OP == OP_GATED_GRAD) {
#pragma unroll
        for (int i = 0; i < E; ++i) { value[i] *= y[i]; slope[i] *= b[i]; }
        zero_outside<G, W>(t, value);
        top_u = max_bits_of<E>(value);
        store_rows<G, W>(D, o.out_kind, rows_at(t, width, N), value, sD, top_u);
    }
#pragma unroll
    for (int i = 0; i < E; ++i) y[i] *= slope[i];
    zero_outside<G, W>(t, y);
    top = max_bits_of<E>(y);
    store_rows<G, W>(D, o.out_kind, rows_at(t, width, 0), y, sD, top);
    return max(top, top_u);
}

// One row of W columns, `left` (>= 1) of them inside, with o.side read here.  PAIR: OP_GATED, else one of the others.
template <int W, bool PAIR>
__device__ __forceinline__ unsigned op_row(const OpArgs& o, void* D, int64_t N, int64_t row, int64_t col, int left, float (&y)[W], float (&u)[W],
                                           const float (&bias)[W], float sD)
{
    float a[W] = {}, b[W] = {};
    const OutRows<1> t = {{row}, col, left, 1u, false};
    if (PAIR) return op_finish<1, W, OP_GATED>(o, D, N, t, y, u, bias, a, b, sD);
    const int64_t width = o.op == OP_GATED_GRAD ? 2 * N : N;
    if (o.side) load_row<W>(o.side, o.side_dtype, row * width + col, left, a);
    if (o.op == OP_ACT) return op_finish<1, W, OP_ACT>(o, D, N, t, y, u, bias, a, b, sD);
    if (o.op == OP_ACT_GRAD) return op_finish<1, W, OP_ACT_GRAD>(o, D, N, t, y, u, bias, a, b, sD);
    load_row<W>(o.side, o.side_dtype, row * width + N + col, left, b);
    return op_finish<1, W, OP_GATED_GRAD>(o, D, N, t, y, u, bias, a, b, sD);
}

// The workgroup's maximum on its way out; `bits`: of the lanes of one wave.
__device__ __forceinline__ void op_commit_top(const OpArgs& o, unsigned bits)
{
    if (!o.tops) { wave_amax_commit(bits, o.amax_out); return; }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) bits = max(bits, (unsigned)__shfl_xor((int)bits, d, 64));
    if (__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)) == 0) o.tops[blockIdx.x] = bits;
}

// One value that is the same for all lanes, by the scalar unit: a wait for it is not a wait for the vector loads in flight.
__device__ __forceinline__ float op_scalar(const float* p) { return *(const __attribute__((address_space(4))) float*)(uintptr_t)p; }

// 1 / the factor of a column of the product (up: of the second projection), in 64 bits: with 1 / sA it is rounded once.
__device__ __forceinline__ double op_column_factor(const OpArgs& o, int64_t N, int64_t col, bool up)
{
    return 1.0 / (double)o.sB_dev[o.b_factors == B_COLUMN ? col + (up ? N : 0) : o.b_factors == B_PAIR && up ? 1 : 0];
}

}  // namespace
}  // namespace fp8mm
