// Declarations shared by the translation units of the GEMM (tiled kernel instances and the
// dispatcher with the generic kernel).
#pragma once

#include "common.hpp"
#include "fp8_decode.hpp"
#include "fp8_encode.hpp"

#include <optional>

namespace fp8mm {

// Output kinds.  The first two are fp8_dtype_t; the FP8 kinds write one byte per output.
enum { OUT_F32 = 0, OUT_BF16 = 1, OUT_E4M3 = 2, OUT_E5M2 = 3 };
inline int out_elem_size(int kind) { return kind == OUT_F32 ? 4 : kind == OUT_BF16 ? 2 : 1; }

// How the products are formed and summed.
//   ACC_F16: operands widened to fp16 (exact for both FP8 formats), fp16 matrix-core
//            instructions.  These sum each instruction's products in a window of at least 24
//            bits: fp32-grade accumulation, at half the FP8 peak rate.
//   ACC_FP8: FP8 matrix-core instructions at the full FP8 rate.  The hardware adds each run of
//            8 products (the 8 bytes of a lane's register pair) after aligning them to the
//            largest and dropping what lies more than 13 bits below its leading bit, then
//            accumulates the runs in fp32.
enum { ACC_F16 = 0, ACC_FP8 = 1 };

// What happens to an accumulator on its way out (Section 2: the scaling factors are taken out
// once per dot product; results may be converted to FP8 before they are written):
//   c_ij = acc_ij / (sA_i * sB_j);  amax = max |c_ij|;  D_ij = cast_out(c_ij * sD)
// sA is one value or one per row of op(A), sB one value or one per column of op(B); sD applies
// to FP8 outputs only.
struct EpilogueArgs {
    float sA, sB;                 // host values, used where the device pointer is null
    const float* sA_dev;          // null, one value, or M values if a_per_row
    const float* sB_dev;          // null, one value, or N values if b_per_col
    const float* sD_dev;          // null (= 1) or one value
    float* amax_out;              // null or one cell, zeroed by the launcher, raised with atomicMax
    int out_kind;
    int a_per_row, b_per_col;
};

struct GemmArgs {
    const uint8_t* A; const uint8_t* B; void* C;
    int64_t M, N, K;
    int fmtA, fmtB;
    bool transA, transB;          // A stored K x M / B stored N x K
    int acc;                      // ACC_*
    int tile_n;                   // width of the tiled kernel's tile: 256, 192 or 128 (chosen by the dispatcher)
    int wide_cols;                // tiled kernel: > 0 = two widths in one launch, this many tile columns of tile_n (256 or 192)
                                  // first, 128-wide tiles for the rest of N (chosen by the dispatcher)
    bool persist;                 // tiled kernel, narrow tile: the persistent form (one workgroup per compute unit walks
                                  // several tiles as one K loop); set by the dispatcher where its conditions hold
    int splits, pairs_per_split;  // tiled kernel only: splits > 1 cuts K into slices of pairs_per_split stage pairs
                                  // (128 bytes each); C is then a workspace of `splits` fp32 M x N matrices
    EpilogueArgs ep;
    hipStream_t stream;
};

// Tiled kernel, one translation unit per (storage orders, accumulation mode):
// layout = 2 * transA + transB.
#define FP8MM_TILED_NAME_(l, a) launch_tiled_l##l##_a##a
#define FP8MM_TILED_NAME(l, a) FP8MM_TILED_NAME_(l, a)
#define FP8MM_DECLARE_TILED(l) \
    int FP8MM_TILED_NAME(l, 0)(const GemmArgs& g); \
    int FP8MM_TILED_NAME(l, 1)(const GemmArgs& g);
FP8MM_DECLARE_TILED(0)
FP8MM_DECLARE_TILED(1)
FP8MM_DECLARE_TILED(2)
FP8MM_DECLARE_TILED(3)
#undef FP8MM_DECLARE_TILED

constexpr int TILE_M = 256, TILE_N = 256, TILE_K = 64;

// The dispatcher's decision for a problem with M, N, K > 0 (what launch_gemm acts on).
enum { GEMM_GENERIC = 1, GEMM_TILED_256 = 2, GEMM_TILED_128 = 3, GEMM_MFMA_ANY = 4, GEMM_TILED_MIXED = 5 };
// small: the form of the small-tile kernel that takes the problem instead (SMALL_*).
// middle: 256 x 192 tiles instead of what `kernel` names; middle_cols > 0: for that many tile columns, 128-wide ones for the rest.
// us: of a problem that the tiled kernel takes, what the model of run times gives for the small-tile form, or for the better of the
// single tile widths.
struct GemmPlan { int kernel; bool elementwise_stores; bool persistent; int wide_cols; int small; bool middle; int middle_cols; double us; };
GemmPlan plan_gemm(const GemmArgs& g, bool whole = true);
// The form (fp8_form_t) of the kernel that launch_gemm takes for it.
int gemm_form(const GemmArgs& g);

int launch_gemm(const GemmArgs& g, const GemmPlan* known = nullptr);      // known: plan_gemm(g, false), where the caller has it

// The matrix-core kernel for any shape and alignment (gemm_mfma_any.hip): operands staged through
// registers; tiles of 256 x 256 or 256 x 128.  Takes every problem with M, N, K > 0 whose tile count fits the grid; the few that its tiles
// do not (see mfma_any_width) run on 64 x 64 tiles of the small-tile kernel.
bool mfma_any_takes(const GemmArgs& g);
int mfma_any_width(const GemmArgs& g);       // 256 or 128 columns; 0: the small-tile kernel
int launch_mfma_any(const GemmArgs& g);
#define FP8MM_ANY_NAME_(l) launch_mfma_any_l##l
#define FP8MM_ANY_NAME(l) FP8MM_ANY_NAME_(l)
int FP8MM_ANY_NAME(0)(const GemmArgs& g, int width);        // one translation unit per pair of storage orders
int FP8MM_ANY_NAME(1)(const GemmArgs& g, int width);
int FP8MM_ANY_NAME(2)(const GemmArgs& g, int width);
int FP8MM_ANY_NAME(3)(const GemmArgs& g, int width);

// The tiled kernel instance for g's storage orders and accumulation mode, with g.tile_n, g.splits,
// g.pairs_per_split as given (the caller has checked that the tiled kernel takes
// the problem).
int launch_tiled(const GemmArgs& g);

// The kernel for small problems (gemm_small.hip), one translation unit per pair of storage orders;
// its forms are named by their output tile; two more of the largest for operands that are both contiguous along K.
enum { SMALL_NONE = -1, SMALL_32x32 = 0, SMALL_32x64 = 1, SMALL_64x64 = 2, SMALL_64x64_LINES8 = 3, SMALL_64x64_LINES4 = 4 };
#define FP8MM_SMALL_NAME_(l) launch_small_l##l
#define FP8MM_SMALL_NAME(l) FP8MM_SMALL_NAME_(l)
int FP8MM_SMALL_NAME(0)(const GemmArgs& g, int form);
int FP8MM_SMALL_NAME(1)(const GemmArgs& g, int form);
int FP8MM_SMALL_NAME(2)(const GemmArgs& g, int form);
int FP8MM_SMALL_NAME(3)(const GemmArgs& g, int form);

// The whole scaled product of a small problem in one launch (scaled_gemm_small.hip), one translation unit per pair of storage orders.  g: the
// product of fp8_scaled_gemm (g.A, g.B: where the operands' FP8 bytes go; factors from scale_out).  launch_scaled_gemm_small sets `took` to
// whether it took the problem (scaled_gemm_small_takes); nothing has been launched where it did not.  plan: of the product, if it was looked for.
constexpr int kScaledSmallLds = 160 * 1024 - 1024;         // dynamic LDS at most (the kernel has a few static words)
constexpr int kScaledSmallRow = 2048;                      // K elements of this many bytes at most
constexpr int kScaledSmallBytes = 192 << 10;               // ... and in all tiles together of fewer than this
int scaled_gemm_small_lds(const GemmArgs& g);
int launch_scaled_gemm_small(const GemmArgs& g, const void* a, const void* b, int in_dtype, float* amax_out, float* scale_out, void* workspace, bool& took,
                             std::optional<GemmPlan>& plan);
#define FP8MM_SCALED_NAME_(l) launch_scaled_gemm_small_l##l
#define FP8MM_SCALED_NAME(l) FP8MM_SCALED_NAME_(l)
#define FP8MM_DECLARE_SCALED(l) \
    int FP8MM_SCALED_NAME(l)(const GemmArgs& g, const void* a, const void* b, int in_dtype, float* amax_out, float* scale_out, void* workspace);
FP8MM_DECLARE_SCALED(0)
FP8MM_DECLARE_SCALED(1)
FP8MM_DECLARE_SCALED(2)
FP8MM_DECLARE_SCALED(3)
#undef FP8MM_DECLARE_SCALED

// Split-K (gemm_splitk.hip): K cut into `splits` slices of pairs_per_split stage pairs.
constexpr int kMaxSplitK = 64;
struct SplitPlan { int splits, pairs_per_split, tile_n; };
SplitPlan plan_splitk(const GemmArgs& g, int requested);
size_t splitk_workspace_bytes(const GemmArgs& g, const SplitPlan& sp);
int launch_gemm_splitk(const GemmArgs& g, const SplitPlan& sp, void* workspace);

// Argument checks shared by the GEMM entry points that take the arguments of fp8_gemm_ex; fills g.
// Returns FP8_OK or the status to return (the error text is set).
int fill_gemm_args(const char* who, GemmArgs& g, const uint8_t* A, int fmtA, int transA, const uint8_t* B, int fmtB,
                   int transB, void* C, int64_t M, int64_t N, int64_t K, int out_dtype, float sA, float sB,
                   const float* sA_dev, const float* sB_dev, int flags, void* stream);

// Microseconds for one tile of the tiled kernel, S stages of 64 along K, as one of several rounds of 256 that
// run at a time (fitted to 4096 x 6144 over K = 512 .. 2048 and to 3294 x 11648 x 4288; within 5 %).  middle: the
// 256 x 192 tile, fitted to 70 products so that it is taken where it is the faster one.
struct TileTimes { double wide, middle, narrow; };
TileTimes tile_times(int acc, double S);
// Time until the last of Tw wide tiles (tw each) and then Tn narrow ones (tn each) ends on 256 units.
double tiles_makespan(int64_t Tw, int64_t Tn, double tw, double tn);

// ---- small device helpers used by the kernels -------------------------------------------------
typedef u32x4 u32x4_any __attribute__((aligned(1)));     // 16 bytes at any address: one load or store on this target

// The vector without its first k bytes (0 <= k < 16), zeros behind the rest.
__device__ __forceinline__ u32x4 drop_bytes(u32x4 v, int k)
{
    if (k & 8) v = (u32x4){v.z, v.w, 0u, 0u};
    if (k & 4) v = (u32x4){v.y, v.z, v.w, 0u};
    const int b = k & 3;
    return (u32x4){__builtin_amdgcn_alignbyte(v.y, v.x, b), __builtin_amdgcn_alignbyte(v.z, v.y, b),
                   __builtin_amdgcn_alignbyte(v.w, v.z, b), __builtin_amdgcn_alignbyte(0u, v.w, b)};
}

// A whole row of fewer than 16 bytes, at the end of the vector.
__device__ __forceinline__ u32x4 load_short(const uint8_t* row, int len)
{
    u32x4 v = {0u, 0u, 0u, 0u};
    for (int j = 0; j < len; ++j) {
        const int at = 16 - len + j;
        const unsigned b = (unsigned)row[j] << (8 * (at & 3));
        v = (u32x4){v.x | (at >> 2 == 0 ? b : 0u), v.y | (at >> 2 == 1 ? b : 0u), v.z | (at >> 2 == 2 ? b : 0u), v.w | (at >> 2 == 3 ? b : 0u)};
    }
    return v;
}

// 16 bytes of a row of `len` bytes, from byte `at` on; zeros beyond the row's end (nothing outside the
// row is read).
__device__ __forceinline__ u32x4 load_guarded(const uint8_t* row, int64_t at, int64_t len)
{
    const int64_t count = len - at;
    if (count >= 16) return *(const u32x4_any*)(row + at);
    if (count <= 0) return (u32x4){0u, 0u, 0u, 0u};
    return drop_bytes(len >= 16 ? *(const u32x4_any*)(row + len - 16) : load_short(row, (int)len), (int)(16 - count));
}

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

// 8 FP8 bytes (two dwords) -> 8 fp16 values, exact (both formats embed in fp16; E4M3's NaN becomes NaN).
template <int FMT>
__device__ __forceinline__ v8h widen8(int lo, int hi)
{
    v2h p0, p1, p2, p3;
    if (FMT == FP8_E4M3) {
        p0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((unsigned)lo, 1.0f, false);
        p1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((unsigned)lo, 1.0f, true);
        p2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((unsigned)hi, 1.0f, false);
        p3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((unsigned)hi, 1.0f, true);
    } else {
        p0 = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8((unsigned)lo, 1.0f, false);
        p1 = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8((unsigned)lo, 1.0f, true);
        p2 = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8((unsigned)hi, 1.0f, false);
        p3 = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8((unsigned)hi, 1.0f, true);
    }
    return (v8h){p0.x, p0.y, p1.x, p1.y, p2.x, p2.y, p3.x, p3.y};
}

__device__ __forceinline__ float scale_value(const float* dev, float host) { return dev ? *dev : host; }

// Largest of `bits` (sign-stripped fp32 patterns; NaN patterns sort above infinity) over the wave,
// then one atomic per wave.
__device__ __forceinline__ void wave_amax_commit(unsigned bits, float* amax_out)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        const unsigned o = (unsigned)__shfl_xor((int)bits, d, 64);
        bits = o > bits ? o : bits;
    }
    // most waves find the cell already large enough and skip the atomic (the lane index comes from
    // the execution mask count, not from threadIdx: nothing has to stay in a register for it)
    if (__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)) == 0 &&
        bits > __hip_atomic_load((unsigned*)amax_out, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT))
        atomicMax((unsigned*)amax_out, bits);
}

}  // namespace fp8mm
