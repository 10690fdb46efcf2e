// extern "C" entry points of the feed-forward operators: argument validation, then one launcher each.
#include "gemm_op.hpp"

using namespace fp8mm;

namespace {

// The checks that the four products share, and their arguments into g and o.  N: columns of D, or of either half of it.
int fill_op(const char* who, GemmArgs& g, OpArgs& o, int op, const uint8_t* A, int fmtA, int transA, const uint8_t* B, int fmtB, int transB, void* D,
            int out_kind, int64_t M, int64_t N, int64_t K, const float* sA_dev, int64_t nsA, const float* sB_dev, int64_t nsB, int act,
            const float* sD_dev, float* amax_out, int flags, void* stream)
{
    clear_error();
    if (flags & ~FP8_GEMM_MFMA8) return fail(FP8_ERR_INVALID_ARG, "%s: unknown flag bits 0x%x", who, flags & ~FP8_GEMM_MFMA8);
    if ((transA != 0 && transA != 1) || (transB != 0 && transB != 1)) return fail(FP8_ERR_INVALID_ARG, "%s: transA/transB must be 0 or 1", who);
    if (!valid_format(fmtA) || !valid_format(fmtB))
        return fail(FP8_ERR_INVALID_ARG, "%s: operand formats (%d, %d) are not fp8_format_t", who, fmtA, fmtB);
    if (out_kind < FP8_OUT_F32 || out_kind > FP8_OUT_E5M2) return fail(FP8_ERR_INVALID_ARG, "%s: out_kind %d is not an fp8_out_t", who, out_kind);
    if (act < FP8_ACT_NONE || act > FP8_ACT_SILU) return fail(FP8_ERR_INVALID_ARG, "%s: act %d is not an fp8_act_t", who, act);
    // (sizes whose byte counts, of a pair of halves in 32 bits, stay within 64 bits)
    constexpr int64_t most = (int64_t)1 << 40;
    if (M < 0 || N < 0 || K < 0) return fail(FP8_ERR_INVALID_ARG, "%s: negative dimension (M=%lld N=%lld K=%lld)", who, (long long)M, (long long)N, (long long)K);
    if (M > most || N > most || K > most || (M > 0 && N > ((int64_t)1 << 58) / M)) return fail(FP8_ERR_UNSUPPORTED, "%s: a dimension or output of more than 2^40 or 2^58", who);
    const int64_t columns = op == OP_GATED ? 2 * N : N;
    if (!sA_dev || !sB_dev) return fail(FP8_ERR_INVALID_ARG, "%s: sA_dev or sB_dev is NULL", who);
    if (nsA != 1 && nsA != M) return fail(FP8_ERR_INVALID_ARG, "%s: nsA = %lld is neither 1 nor M", who, (long long)nsA);
    const bool pair = op == OP_GATED && nsB == 2;
    if (nsB != 1 && nsB != columns && !pair)
        return fail(FP8_ERR_INVALID_ARG, op == OP_GATED ? "%s: nsB = %lld is neither 1, 2 nor 2F" : "%s: nsB = %lld is neither 1 nor the columns of op(B)", who, (long long)nsB);
    if (((uintptr_t)sA_dev | (uintptr_t)sB_dev | (uintptr_t)sD_dev | (uintptr_t)amax_out) % 4)
        return fail(FP8_ERR_INVALID_ARG, "%s: a scale or amax pointer is misaligned", who);
    if (sD_dev && out_kind < FP8_OUT_E4M3) return fail(FP8_ERR_INVALID_ARG, "%s: an output factor applies to FP8 outputs only", who);
    if (M > 0 && N > 0) {
        if (!D) return fail(FP8_ERR_INVALID_ARG, "%s: the output is NULL", who);
        if (K > 0 && (!A || !B)) return fail(FP8_ERR_INVALID_ARG, "%s: A or B is NULL", who);
        if ((uintptr_t)D % (uintptr_t)out_elem_size(out_kind)) return fail(FP8_ERR_INVALID_ARG, "%s: the output is not aligned to its element size", who);
    }
    g = GemmArgs{};
    g.A = A; g.B = B; g.C = D; g.M = M; g.N = N; g.K = K; g.fmtA = fmtA; g.fmtB = fmtB;
    g.transA = transA != 0; g.transB = transB != 0; g.acc = (flags & FP8_GEMM_MFMA8) ? ACC_FP8 : ACC_F16;
    g.splits = 1;
    g.stream = (hipStream_t)stream;
    o = OpArgs{};
    o.sA_dev = sA_dev; o.sB_dev = sB_dev; o.sD_dev = sD_dev; o.amax_out = amax_out;
    o.op = op; o.act = act; o.out_kind = out_kind;
    o.a_per_row = nsA == M && M != 1;
    o.b_factors = nsB == 1 ? B_ONE : pair ? B_PAIR : B_COLUMN;
    return FP8_OK;
}

// A tensor beside the product: its type, alignment and presence.
int check_side(const char* who, const char* name, const void* p, int dtype, bool required)
{
    if (!p) return required ? fail(FP8_ERR_INVALID_ARG, "%s: %s is NULL", who, name) : (int)FP8_OK;
    if (!valid_dtype(dtype)) return fail(FP8_ERR_INVALID_ARG, "%s: the type %d of %s is not an fp8_dtype_t", who, dtype, name);
    if ((uintptr_t)p % (dtype == FP8_F32 ? 4 : 2)) return fail(FP8_ERR_INVALID_ARG, "%s: %s is not aligned to its element size", who, name);
    return FP8_OK;
}

// Bytes of a matrix; one that no memory holds counts as 2^61.
int64_t bytes_of(int64_t rows, int64_t cols, int size)
{
    constexpr int64_t most = (int64_t)1 << 61;
    return rows > 0 && cols > 0 && rows > most / cols / size ? most : rows * cols * size;
}

// Whether np bytes from p on and nq from q on share memory.
bool overlap(const void* p, int64_t np, const void* q, int64_t nq) { return p && q && (uintptr_t)p < (uintptr_t)q + nq && (uintptr_t)q < (uintptr_t)p + np; }

int check_tensors(const char* who, int count, const void* const* x, const size_t* n, const int* dtype)
{
    if (count < 0) return fail(FP8_ERR_INVALID_ARG, "%s: count %d is negative", who, count);
    if (count > 0 && (!x || !n || !dtype)) return fail(FP8_ERR_INVALID_ARG, "%s: x, n or dtype is NULL", who);
    for (int i = 0; i < count; ++i) {
        if (!valid_dtype(dtype[i])) return fail(FP8_ERR_INVALID_ARG, "%s: dtype[%d] = %d is not an fp8_dtype_t", who, i, dtype[i]);
        if (n[i] > (size_t)1 << 45) return fail(FP8_ERR_UNSUPPORTED, "%s: tensor %d has more than 2^45 elements", who, i);
        if (n[i] > 0 && !x[i]) return fail(FP8_ERR_INVALID_ARG, "%s: x[%d] is NULL with n = %zu", who, i, n[i]);
        if (n[i] > 0 && (uintptr_t)x[i] % (dtype[i] == FP8_F32 ? 4 : 2)) return fail(FP8_ERR_INVALID_ARG, "%s: x[%d] is not aligned to its element size", who, i);
    }
    return FP8_OK;
}

}  // namespace

extern "C" {

int fp8_gemm_act(const uint8_t* A, int fmtA, int transA, const uint8_t* B, int fmtB, int transB, void* D, int out_kind, int64_t M, int64_t N, int64_t K,
                 const float* sA_dev, int64_t nsA, const float* sB_dev, int64_t nsB, int act, const void* bias, int bias_dtype,
                 const void* residual, int residual_dtype, void* Z, int Z_dtype, const float* sD_dev, float* amax_out, int flags, void* stream)
{
    const char* who = "fp8_gemm_act";
    GemmArgs g; OpArgs o;
    if (int e = fill_op(who, g, o, OP_ACT, A, fmtA, transA, B, fmtB, transB, D, out_kind, M, N, K, sA_dev, nsA, sB_dev, nsB, act, sD_dev, amax_out, flags, stream)) return e;
    if (int e = check_side(who, "bias", bias, bias_dtype, false)) return e;
    if (int e = check_side(who, "residual", residual, residual_dtype, false)) return e;
    if (int e = check_side(who, "Z", Z, Z_dtype, false)) return e;
    const int64_t d_bytes = bytes_of(M, N, out_elem_size(out_kind)), r_bytes = bytes_of(M, N, out_elem_size(residual_dtype)), z_bytes = bytes_of(M, N, out_elem_size(Z_dtype));
    if (overlap(D, d_bytes, residual, r_bytes) && (D != residual || out_kind != residual_dtype))
        return fail(FP8_ERR_INVALID_ARG, "%s: residual overlaps D, whose start or type is another", who);
    if (overlap(Z, z_bytes, D, d_bytes) || overlap(Z, z_bytes, residual, r_bytes) || overlap(Z, z_bytes, A, bytes_of(M, K, 1)) || overlap(Z, z_bytes, B, bytes_of(K, N, 1)))
        return fail(FP8_ERR_INVALID_ARG, "%s: Z overlaps another argument", who);
    o.bias = bias; o.bias_dtype = bias_dtype; o.side = residual; o.side_dtype = residual_dtype; o.kept = Z; o.kept_dtype = Z_dtype;
    return launch_gemm_op(g, o, nullptr);
}

size_t fp8_gemm_act_grad_workspace_size(int64_t M, int64_t N)
{
    if (M <= 0 || N <= 0) return 0;
    const size_t rows = (size_t)(M - 1) / kOpSumRows + 1;
    return rows > SIZE_MAX / 4 / (size_t)N ? SIZE_MAX : rows * (size_t)N * 4;
}

int fp8_gemm_act_grad(const uint8_t* A, int fmtA, int transA, const uint8_t* B, int fmtB, int transB, void* D, int out_kind, int64_t M, int64_t N, int64_t K,
                      const float* sA_dev, int64_t nsA, const float* sB_dev, int64_t nsB, int act, const void* Z, int Z_dtype, float* dbias,
                      void* workspace, size_t workspace_bytes, const float* sD_dev, float* amax_out, int flags, void* stream)
{
    const char* who = "fp8_gemm_act_grad";
    GemmArgs g; OpArgs o;
    if (int e = fill_op(who, g, o, OP_ACT_GRAD, A, fmtA, transA, B, fmtB, transB, D, out_kind, M, N, K, sA_dev, nsA, sB_dev, nsB, act, sD_dev, amax_out, flags, stream)) return e;
    if (int e = check_side(who, "Z", Z, Z_dtype, M > 0 && N > 0)) return e;
    if (Z && overlap(D, bytes_of(M, N, out_elem_size(out_kind)), Z, bytes_of(M, N, out_elem_size(Z_dtype))) && (D != Z || out_kind != Z_dtype))
        return fail(FP8_ERR_INVALID_ARG, "%s: Z overlaps D, whose start or type is another", who);
    if (dbias) {
        const size_t need = fp8_gemm_act_grad_workspace_size(M, N);
        if ((uintptr_t)dbias % 4) return fail(FP8_ERR_INVALID_ARG, "%s: dbias is misaligned", who);
        if (need > 0 && (!workspace || (uintptr_t)workspace % 4 || workspace_bytes < need))
            return fail(FP8_ERR_INVALID_ARG, "%s: the workspace is NULL, misaligned or smaller than %zu bytes", who, need);
        o.sums = (float*)workspace;
    }
    o.side = Z; o.side_dtype = Z_dtype;
    return launch_gemm_op(g, o, dbias);
}

int fp8_gemm_gated(const uint8_t* A, int fmtA, int transA, const uint8_t* B, int fmtB, int transB, void* H, int out_kind, int64_t M, int64_t F, int64_t K,
                   const float* sA_dev, int64_t nsA, const float* sB_dev, int64_t nsB, int act, void* GU, int GU_dtype,
                   const float* sH_dev, float* amax_out, int flags, void* stream)
{
    const char* who = "fp8_gemm_gated";
    GemmArgs g; OpArgs o;
    if (int e = fill_op(who, g, o, OP_GATED, A, fmtA, transA, B, fmtB, transB, H, out_kind, M, F, K, sA_dev, nsA, sB_dev, nsB, act, sH_dev, amax_out, flags, stream)) return e;
    if (int e = check_side(who, "GU", GU, GU_dtype, false)) return e;
    const int64_t gu_bytes = bytes_of(M, 2 * F, out_elem_size(GU_dtype));
    if (overlap(GU, gu_bytes, H, bytes_of(M, F, out_elem_size(out_kind))) || overlap(GU, gu_bytes, A, bytes_of(M, K, 1)) || overlap(GU, gu_bytes, B, bytes_of(K, 2 * F, 1)))
        return fail(FP8_ERR_INVALID_ARG, "%s: GU overlaps another argument", who);
    o.kept = GU; o.kept_dtype = GU_dtype;
    return launch_gemm_op(g, o, nullptr);
}

int fp8_gemm_gated_grad(const uint8_t* A, int fmtA, int transA, const uint8_t* B, int fmtB, int transB, void* dGU, int out_kind, int64_t M, int64_t F, int64_t K,
                        const float* sA_dev, int64_t nsA, const float* sB_dev, int64_t nsB, int act, const void* GU, int GU_dtype,
                        const float* sD_dev, float* amax_out, int flags, void* stream)
{
    const char* who = "fp8_gemm_gated_grad";
    GemmArgs g; OpArgs o;
    if (int e = fill_op(who, g, o, OP_GATED_GRAD, A, fmtA, transA, B, fmtB, transB, dGU, out_kind, M, F, K, sA_dev, nsA, sB_dev, nsB, act, sD_dev, amax_out, flags, stream)) return e;
    if (int e = check_side(who, "GU", GU, GU_dtype, M > 0 && F > 0)) return e;
    if (GU && overlap(dGU, bytes_of(M, 2 * F, out_elem_size(out_kind)), GU, bytes_of(M, 2 * F, out_elem_size(GU_dtype))) && (dGU != GU || out_kind != GU_dtype))
        return fail(FP8_ERR_INVALID_ARG, "%s: GU overlaps dGU, whose start or type is another", who);
    o.side = GU; o.side_dtype = GU_dtype;
    return launch_gemm_op(g, o, nullptr);
}

int fp8_grad_norm(int count, const void* const* x, const size_t* n, const int* dtype, float* norm_out, void* workspace, void* stream)
{
    const char* who = "fp8_grad_norm";
    clear_error();
    if (int e = check_tensors(who, count, x, n, dtype)) return e;
    if (!norm_out || (uintptr_t)norm_out % 4) return fail(FP8_ERR_INVALID_ARG, "%s: norm_out is NULL or misaligned", who);
    if (!workspace || (uintptr_t)workspace % 8) return fail(FP8_ERR_INVALID_ARG, "%s: workspace is NULL or misaligned", who);
    return launch_grad_norm(count, x, n, dtype, norm_out, workspace, (hipStream_t)stream);
}

int fp8_grad_clip(int count, const void* const* x, const size_t* n, const int* dtype, void* const* out, const float* norm, float max_norm, void* stream)
{
    const char* who = "fp8_grad_clip";
    clear_error();
    if (int e = check_tensors(who, count, x, n, dtype)) return e;
    if (!norm || (uintptr_t)norm % 4) return fail(FP8_ERR_INVALID_ARG, "%s: norm is NULL or misaligned", who);
    if (!(max_norm >= 0.0f)) return fail(FP8_ERR_INVALID_ARG, "%s: max_norm is negative or NaN", who);
    if (out)
        for (int i = 0; i < count; ++i) {
            if (n[i] == 0) continue;
            const int64_t bytes = (int64_t)n[i] * (dtype[i] == FP8_F32 ? 4 : 2);
            if (!out[i]) return fail(FP8_ERR_INVALID_ARG, "%s: out[%d] is NULL with n = %zu", who, i, n[i]);
            if ((uintptr_t)out[i] % (dtype[i] == FP8_F32 ? 4 : 2)) return fail(FP8_ERR_INVALID_ARG, "%s: out[%d] is not aligned to its element size", who, i);
            if (out[i] != x[i] && overlap(out[i], bytes, x[i], bytes)) return fail(FP8_ERR_INVALID_ARG, "%s: out[%d] overlaps x[%d] in part", who, i, i);
        }
    return launch_grad_clip(count, x, n, dtype, out ? out : (void* const*)x, norm, max_norm, (hipStream_t)stream);
}

}  // extern "C"
