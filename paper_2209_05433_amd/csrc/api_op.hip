// extern "C" entry points of the feed-forward operators, the loss over a vocabulary and AdamW: argument validation, then one launcher each.
#include "gemm_loss.hpp"

#include <algorithm>
#include <cstdio>
#include <exception>
#include <vector>

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
    o.sA_dev = sA_dev; o.sB_dev = sB_dev; o.sD_dev = sD_dev; o.amax_out = amax_out;
    o.op = op; o.act = act; o.out_kind = out_kind;
    o.a_per_row = nsA == M && M != 1;
    o.b_factors = nsB == 1 ? B_ONE : pair ? B_PAIR : B_COLUMN;
    return FP8_OK;
}

// What the loss and its gradient share beyond that.
int fill_loss(const char* who, LossArgs& o, int64_t M, const int64_t* labels, int64_t first, float z_weight)
{
    if (M > 0 && (!labels || (uintptr_t)labels % 8)) return fail(FP8_ERR_INVALID_ARG, "%s: labels is NULL or misaligned", who);
    if (first < 0) return fail(FP8_ERR_INVALID_ARG, "%s: first = %lld is negative", who, (long long)first);
    if (!(z_weight >= 0.0f && z_weight < __builtin_inff())) return fail(FP8_ERR_INVALID_ARG, "%s: z_weight is negative or not finite", who);
    o.labels = labels; o.first = first; o.z_weight = z_weight;
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
bool overlap(const void* p, int64_t np, const void* q, int64_t nq) { return p && q && np > 0 && nq > 0 && (uintptr_t)p < (uintptr_t)q + nq && (uintptr_t)q < (uintptr_t)p + np; }

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

// What a step writes must be nothing else that it reads or writes, of the same tensor or another (tied weights that are in the list twice would be updated by
// two workgroups at once).  Sorted by address, neither a range that is written may begin before the end of any other one, nor any range before the end of one that is written.
struct MemoryRange { uintptr_t begin, end; int kind, index; };
const char* const kAdamMemory[] = {"p", "g", "m", "v", "q", "m_scale", "v_scale", "lr", "step", "norm", "q_scale", "q_amax"};
int check_adamw_memory(const char* who, int count, void* const* p, const int* p_dtype, const void* const* g, const int* g_dtype, const size_t* n, void* const* m, void* const* v,
                       bool states8, float* const* m_scale, float* const* v_scale, uint8_t* const* q, const float* lr, const int64_t* step, const float* norm, const float* q_scale,
                       const float* q_amax)
{
    std::vector<MemoryRange> all, merged;
    try {
        const size_t most = (size_t)std::max(count, 0) * (states8 ? 7 : 5) + 5;
        all.reserve(most);
        merged.reserve(most);
        // one list of tensors behind the other: each is in the order of its addresses already as a rule, and joined to those before by a merge
        auto add = [&](int kind, auto begin_of, auto bytes_of_each) {
            const size_t first = all.size();
            for (int i = 0; i < count; ++i) {
                const uintptr_t at = n[i] ? (uintptr_t)begin_of(i) : 0;
                if (at) all.push_back({at, at + bytes_of_each(i), kind, i});
            }
            auto less = [](const MemoryRange& a, const MemoryRange& b) { return a.begin < b.begin; };
            if (!std::is_sorted(all.begin() + first, all.end(), less)) std::sort(all.begin() + first, all.end(), less);
            if (first == 0 || first == all.size() || !less(all[first], all[first - 1])) return;
            merged.resize(all.size());
            std::merge(all.begin(), all.begin() + first, all.begin() + first, all.end(), merged.begin(), less);
            all.swap(merged);
        };
        auto blocks = [&](int i) { return 4 * ((n[i] + FP8_STATE_BLOCK - 1) / FP8_STATE_BLOCK); };
        const size_t state = states8 ? 1 : 4;
        add(0, [&](int i) { return p[i]; }, [&](int i) { return n[i] * (p_dtype[i] == FP8_F32 ? 4 : 2); });
        add(1, [&](int i) { return g[i]; }, [&](int i) { return n[i] * (g_dtype[i] == FP8_F32 ? 4 : 2); });
        add(2, [&](int i) { return m[i]; }, [&](int i) { return n[i] * state; });
        add(3, [&](int i) { return v[i]; }, [&](int i) { return n[i] * state; });
        if (q) add(4, [&](int i) { return q[i]; }, [&](int i) { return n[i]; });
        if (states8) add(5, [&](int i) { return m_scale[i]; }, blocks);
        if (states8) add(6, [&](int i) { return v_scale[i]; }, blocks);
        if (all.empty()) return FP8_OK;
        const struct { const void* p; size_t bytes; } single[] = {{lr, 4}, {step, 8}, {norm, 4}, {q ? q_scale : nullptr, 4 * (size_t)count}, {q_amax, 4 * (size_t)count}};
        for (int k = 0; k < 5; ++k) {
            if (!single[k].p) continue;
            const MemoryRange x = {(uintptr_t)single[k].p, (uintptr_t)single[k].p + single[k].bytes, 7 + k, -1};
            all.insert(std::upper_bound(all.begin(), all.end(), x, [](const MemoryRange& a, const MemoryRange& b) { return a.begin < b.begin; }), x);
        }
    } catch (const std::exception&) {
        return fail(FP8_ERR_UNSUPPORTED, "%s: no host memory for a list of %d tensors", who, count);
    }
    auto written = [](const MemoryRange& x) { return x.kind != 1 && x.kind < 7; };
    auto named = [](const MemoryRange& x, char (&to)[32]) {
        if (x.index < 0) std::snprintf(to, sizeof to, "%s", kAdamMemory[x.kind]);
        else std::snprintf(to, sizeof to, "%s[%d]", kAdamMemory[x.kind], x.index);
        return to;
    };
    char one[32], two[32];
    const MemoryRange* furthest = nullptr;                 // of those before
    const MemoryRange* furthest_written = nullptr;
    for (const MemoryRange& x : all) {
        const MemoryRange* other = written(x) ? furthest : furthest_written;
        if (other && x.begin < other->end)
            return fail(FP8_ERR_INVALID_ARG, "%s: %s%s and %s overlap", who, x.kind == 0 && other->kind == 0 ? "two of the weights, " : "", named(*other, one), named(x, two));
        if (!furthest || x.end > furthest->end) furthest = &x;
        if (written(x) && (!furthest_written || x.end > furthest_written->end)) furthest_written = &x;
    }
    // (the maxima: no tensor that is written holds them, as seen above, nor a gradient)
    for (int i = 0; q_amax && i < count; ++i)
        if (n[i] && overlap(q_amax, 4 * (int64_t)count, g[i], (int64_t)n[i] * (g_dtype[i] == FP8_F32 ? 4 : 2))) return fail(FP8_ERR_INVALID_ARG, "%s: g[%d] and q_amax overlap", who, i);
    return FP8_OK;
}

}  // namespace

extern "C" {

int fp8_gemm_act(const uint8_t* A, int fmtA, int transA, const uint8_t* B, int fmtB, int transB, void* D, int out_kind, int64_t M, int64_t N, int64_t K,
                 const float* sA_dev, int64_t nsA, const float* sB_dev, int64_t nsB, int act, const void* bias, int bias_dtype,
                 const void* residual, int residual_dtype, void* Z, int Z_dtype, const float* sD_dev, float* amax_out, int flags, void* stream)
{
    const char* who = "fp8_gemm_act";
    GemmArgs g; OpArgs o{};
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
    GemmArgs g; OpArgs o{};
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
    GemmArgs g; OpArgs o{};
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
    GemmArgs g; OpArgs o{};
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

size_t fp8_gemm_xent_workspace_size(int64_t M, int64_t N)
{
    if (M <= 0 || N < 0) return 0;
    const size_t rows = (size_t)N / 32 + (N % 32 != 0) + 1;
    return rows > SIZE_MAX / 8 / (size_t)M ? SIZE_MAX : rows * (size_t)M * 8;
}

int fp8_gemm_xent(const uint8_t* A, int fmtA, int transA, const uint8_t* B, int fmtB, int transB, int64_t M, int64_t N, int64_t K,
                  const float* sA_dev, int64_t nsA, const float* sB_dev, int64_t nsB, const int64_t* labels, int64_t first, float z_weight,
                  float* loss, float* lse, void* workspace, size_t workspace_bytes, int flags, void* stream)
{
    const char* who = "fp8_gemm_xent";
    GemmArgs g; LossArgs o{};
    // (no output of the product: the place of one that passes the checks)
    if (int e = fill_op(who, g, o, OP_LOSS, A, fmtA, transA, B, fmtB, transB, lse, FP8_OUT_F32, M, N, K, sA_dev, nsA, sB_dev, nsB, FP8_ACT_NONE, nullptr, nullptr, flags, stream)) return e;
    if (int e = fill_loss(who, o, M, labels, first, z_weight)) return e;
    if (M == 0) return FP8_OK;
    if (!loss || !lse || ((uintptr_t)loss | (uintptr_t)lse) % 4) return fail(FP8_ERR_INVALID_ARG, "%s: loss or lse is NULL or misaligned", who);
    const size_t need = fp8_gemm_xent_workspace_size(M, N);
    if (!workspace || (uintptr_t)workspace % 8 || workspace_bytes < need)
        return fail(FP8_ERR_INVALID_ARG, "%s: the workspace is NULL, misaligned or smaller than %zu bytes", who, need);
    const int64_t cells = 4 * M;
    if (overlap(loss, cells, lse, cells) || overlap(loss, cells, workspace, (int64_t)need) || overlap(lse, cells, workspace, (int64_t)need) ||
        overlap(labels, 8 * M, loss, cells) || overlap(labels, 8 * M, lse, cells) || overlap(labels, 8 * M, workspace, (int64_t)need))
        return fail(FP8_ERR_INVALID_ARG, "%s: loss, lse, the workspace and labels overlap", who);
    const struct { const void* p; int64_t bytes; } in[] = {{A, bytes_of(M, K, 1)}, {B, bytes_of(K, N, 1)}, {sA_dev, 4 * nsA}, {sB_dev, 4 * nsB}};
    for (const auto& x : in)
        if (overlap(loss, cells, x.p, x.bytes) || overlap(lse, cells, x.p, x.bytes) || overlap(workspace, (int64_t)need, x.p, x.bytes))
            return fail(FP8_ERR_INVALID_ARG, "%s: loss, lse or the workspace overlaps an operand or its factors", who);
    o.partials = workspace;
    return launch_gemm_loss(g, o, loss, lse);
}

int fp8_gemm_xent_grad(const uint8_t* A, int fmtA, int transA, const uint8_t* B, int fmtB, int transB, void* D, int out_kind, int64_t M, int64_t N, int64_t K,
                       const float* sA_dev, int64_t nsA, const float* sB_dev, int64_t nsB, const int64_t* labels, int64_t first, float z_weight,
                       const float* lse, const float* dloss, int64_t ndloss, const float* sD_dev, float* amax_out, int flags, void* stream)
{
    const char* who = "fp8_gemm_xent_grad";
    GemmArgs g; LossArgs o{};
    if (int e = fill_op(who, g, o, OP_LOSS_GRAD, A, fmtA, transA, B, fmtB, transB, D, out_kind, M, N, K, sA_dev, nsA, sB_dev, nsB, FP8_ACT_NONE, sD_dev, amax_out, flags, stream)) return e;
    if (int e = fill_loss(who, o, M, labels, first, z_weight)) return e;
    if (ndloss != 1 && ndloss != M) return fail(FP8_ERR_INVALID_ARG, "%s: ndloss = %lld is neither 1 nor M", who, (long long)ndloss);
    if (M > 0 && (!lse || !dloss || ((uintptr_t)lse | (uintptr_t)dloss) % 4)) return fail(FP8_ERR_INVALID_ARG, "%s: lse or dloss is NULL or misaligned", who);
    const int64_t d_bytes = bytes_of(M, N, out_elem_size(out_kind));
    const struct { const void* p; int64_t bytes; } in[] = {{A, bytes_of(M, K, 1)}, {B, bytes_of(K, N, 1)}, {labels, 8 * M}, {lse, 4 * M}, {dloss, 4 * ndloss}, {sA_dev, 4 * nsA},
                                                           {sB_dev, 4 * nsB}, {sD_dev, 4}, {amax_out, 4}};
    for (const auto& x : in)
        if (overlap(D, d_bytes, x.p, x.bytes)) return fail(FP8_ERR_INVALID_ARG, "%s: D overlaps another argument", who);
    for (int i = 0; i < 4; ++i)
        if (overlap(amax_out, 4, in[i].p, in[i].bytes)) return fail(FP8_ERR_INVALID_ARG, "%s: amax_out overlaps an operand, labels or lse", who);
    o.lse = lse; o.dloss = dloss; o.dloss_per_row = ndloss == M && M != 1;
    return launch_gemm_loss(g, o, nullptr, nullptr);
}

int fp8_adamw(int count, void* const* p, const int* p_dtype, const void* const* g, const int* g_dtype, const size_t* n, void* const* m, void* const* v,
              int state_kind, float* const* m_scale, float* const* v_scale, uint64_t seed, const float* weight_decay, const float* lr, const int64_t* step,
              double beta1, double beta2, float eps, const float* norm, float max_norm, uint8_t* const* q, int q_fmt, const float* q_scale, float* q_amax,
              int flags, void* stream)
{
    const char* who = "fp8_adamw";
    clear_error();
    if (flags & ~FP8_ADAMW_SKIP_NONFINITE) return fail(FP8_ERR_INVALID_ARG, "%s: unknown flag bits 0x%x", who, flags & ~FP8_ADAMW_SKIP_NONFINITE);
    if (state_kind != FP8_STATE_F32 && state_kind != FP8_STATE_FP8) return fail(FP8_ERR_INVALID_ARG, "%s: state_kind %d is not an fp8_state_t", who, state_kind);
    const bool states8 = state_kind == FP8_STATE_FP8;
    if (int e = check_tensors(who, count, (const void* const*)p, n, p_dtype)) return e;
    if (int e = check_tensors(who, count, g, n, g_dtype)) return e;
    if (count > 0 && (!m || !v || (states8 && (!m_scale || !v_scale)))) return fail(FP8_ERR_INVALID_ARG, "%s: a list of states is NULL", who);
    if (!lr || (uintptr_t)lr % 4 || !step || (uintptr_t)step % 8) return fail(FP8_ERR_INVALID_ARG, "%s: lr or step is NULL or misaligned", who);
    if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0)) return fail(FP8_ERR_INVALID_ARG, "%s: beta1 or beta2 lies outside [0, 1)", who);
    if (!(eps >= 0.0f && eps < __builtin_inff())) return fail(FP8_ERR_INVALID_ARG, "%s: eps is negative or not finite", who);
    if ((uintptr_t)norm % 4) return fail(FP8_ERR_INVALID_ARG, "%s: norm is misaligned", who);
    if (norm && !(max_norm >= 0.0f)) return fail(FP8_ERR_INVALID_ARG, "%s: max_norm is negative or NaN", who);
    if (q && !valid_format(q_fmt)) return fail(FP8_ERR_INVALID_ARG, "%s: q_fmt %d is not an fp8_format_t", who, q_fmt);
    if (q && count > 0 && !q_scale) return fail(FP8_ERR_INVALID_ARG, "%s: q_scale is NULL", who);
    if (((uintptr_t)q_scale | (uintptr_t)q_amax) % 4) return fail(FP8_ERR_INVALID_ARG, "%s: q_scale or q_amax is misaligned", who);
    for (int i = 0; i < count; ++i) {
        if (weight_decay && !(weight_decay[i] >= 0.0f && weight_decay[i] < __builtin_inff()))
            return fail(FP8_ERR_INVALID_ARG, "%s: weight_decay[%d] is negative or not finite", who, i);
        if (n[i] > (size_t)1 << 43) return fail(FP8_ERR_UNSUPPORTED, "%s: tensor %d has more than 2^43 elements", who, i);
        if (n[i] == 0) continue;
        const int state = states8 ? 1 : 4;
        if (!m[i] || !v[i] || (uintptr_t)m[i] % state || (uintptr_t)v[i] % state) return fail(FP8_ERR_INVALID_ARG, "%s: m[%d] or v[%d] is NULL or misaligned", who, i, i);
        if (states8 && (!m_scale[i] || !v_scale[i] || ((uintptr_t)m_scale[i] | (uintptr_t)v_scale[i]) % 4))
            return fail(FP8_ERR_INVALID_ARG, "%s: m_scale[%d] or v_scale[%d] is NULL or misaligned", who, i, i);
    }
    if (int e = check_adamw_memory(who, count, p, p_dtype, g, g_dtype, n, m, v, states8, m_scale, v_scale, q, lr, step, norm, q_scale, q_amax)) return e;
    AdamwArgs a{};
    a.count = count; a.p = p; a.p_dtype = p_dtype; a.g = g; a.g_dtype = g_dtype; a.n = n; a.m = m; a.v = v;
    a.states8 = states8; a.m_scale = m_scale; a.v_scale = v_scale; a.seed = seed;
    a.weight_decay = weight_decay; a.lr = lr; a.step = step; a.beta1 = beta1; a.beta2 = beta2; a.eps = eps;
    a.norm = norm; a.max_norm = max_norm; a.q = q; a.q_fmt = q_fmt; a.q_scale = q_scale; a.q_amax = q_amax;
    a.skip_nonfinite = (flags & FP8_ADAMW_SKIP_NONFINITE) != 0;
    a.stream = (hipStream_t)stream;
    return launch_adamw(a);
}

}  // extern "C"
