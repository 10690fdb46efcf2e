/* Host-side exercise of the feed-forward operators and the gradient calls, for a build of the library with AddressSanitizer and
 * UndefinedBehaviorSanitizer on the host code (tests/test_op_sanitizers.py): their argument checks, workspace sizes, choice of kernels over
 * a seeded sweep of shapes up to 2^36, and the lists of tensors that go into launches.  Launches are recorded and run nothing
 * (tests/hip_recording_stub.c).  Exit status 0 and "ok" on stdout if every call returned what it should. */
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "fp8mm.h"

extern unsigned long long recorded_launches, recorded_workgroups;

static int failures = 0;

#define EXPECT(call, want)                                                                          \
    do {                                                                                            \
        long long got_ = (long long)(call);                                                         \
        if (got_ != (long long)(want)) {                                                            \
            printf("line %d: %s returned %lld, expected %lld (%s)\n", __LINE__, #call, got_,        \
                   (long long)(want), fp8_last_error());                                            \
            ++failures;                                                                             \
        }                                                                                           \
    } while (0)

/* a call, and how many launches and workgroups it takes */
#define LAUNCHES(call, want, n, groups)                                                             \
    do {                                                                                            \
        recorded_launches = recorded_workgroups = 0;                                                \
        EXPECT(call, want);                                                                         \
        EXPECT(recorded_launches, n);                                                               \
        if ((groups) >= 0) EXPECT(recorded_workgroups, groups);                                     \
    } while (0)

#define BAD FP8_ERR_INVALID_ARG

/* stand-ins for device pointers, far apart: never dereferenced on the host */
#define AT(k) ((uintptr_t)(k) << 43)
#define A ((const uint8_t*)AT(1))
#define B ((const uint8_t*)AT(2))
#define D ((void*)AT(3))
#define F ((float*)AT(4))
#define S ((void*)AT(5))
#define Z ((void*)AT(6))

static uint64_t seed = 12345;
static uint64_t draw(void) { seed = seed * 6364136223846793005ull + 1442695040888963407ull; return seed >> 24; }
static int64_t draw_size(int most_bits)
{
    const int bits = (int)(draw() % (uint64_t)(most_bits + 1));
    const int64_t v = (int64_t)(((uint64_t)1 << bits) + (draw() & (((uint64_t)1 << bits) - 1)));
    switch (draw() % 4) { case 0: return v; case 1: return (v + 15) / 16 * 16; case 2: return (v + 255) / 256 * 256; default: return v > 3 ? v - 1 : v; }
}

static void refusals(void)
{
    uint8_t* const Dodd = (uint8_t*)D + 1;
    EXPECT(fp8_gemm_act(A, 2, 0, B, 0, 1, D, 1, 8, 16, 32, F, 1, F, 1, 2, NULL, 0, NULL, 0, NULL, 0, NULL, NULL, 0, NULL), BAD);
    EXPECT(fp8_gemm_act(A, 0, 0, B, 0, 1, Dodd, 1, 8, 16, 32, F, 1, F, 1, 2, NULL, 0, NULL, 0, NULL, 0, NULL, NULL, 0, NULL), BAD);
    EXPECT(fp8_gemm_act(A, 0, 0, B, 0, 1, D, 1, 8, 16, 32, F, 1, F, 1, 5, NULL, 0, NULL, 0, NULL, 0, NULL, NULL, 0, NULL), BAD);
    EXPECT(fp8_gemm_act(A, 0, 0, B, 0, 1, D, 1, 8, 16, 32, F, 3, F, 1, 2, NULL, 0, NULL, 0, NULL, 0, NULL, NULL, 0, NULL), BAD);
    EXPECT(fp8_gemm_act(A, 0, 0, B, 0, 1, D, 1, 8, 16, 32, F, 1, F, 1, 2, (char*)S + 1, 1, NULL, 0, NULL, 0, NULL, NULL, 0, NULL), BAD);
    EXPECT(fp8_gemm_act(A, 0, 0, B, 0, 1, D, 1, 8, 16, 32, F, 1, F, 1, 2, NULL, 0, (char*)D + 2, 1, NULL, 0, NULL, NULL, 0, NULL), BAD);
    EXPECT(fp8_gemm_act(A, 0, 0, B, 0, 1, D, 1, 8, 16, 32, F, 1, F, 1, 2, NULL, 0, NULL, 0, (void*)A, 1, NULL, NULL, 0, NULL), BAD);
    EXPECT(fp8_gemm_act(A, 0, 0, B, 0, 1, D, 1, 8, 16, 32, F, 1, F, 1, 2, NULL, 77, NULL, -5, NULL, 99, NULL, NULL, 0, NULL), FP8_OK);     /* (types of what is NULL) */
    EXPECT(strlen(fp8_last_error()), 0);
    EXPECT(fp8_gemm_act(A, 0, 0, B, 0, 1, D, 1, (int64_t)1 << 41, 1, 1, F, 1, F, 1, 2, NULL, 0, NULL, 0, NULL, 0, NULL, NULL, 0, NULL), FP8_ERR_UNSUPPORTED);
    EXPECT(fp8_gemm_act(A, 0, 0, B, 0, 1, D, 1, INT64_MAX, INT64_MAX, INT64_MAX, F, 1, F, 1, 2, NULL, 0, NULL, 0, NULL, 0, NULL, NULL, 0, NULL), FP8_ERR_UNSUPPORTED);
    EXPECT(fp8_gemm_act(A, 0, 0, B, 0, 1, D, 1, INT64_MIN, 1, 1, F, 1, F, 1, 2, NULL, 0, NULL, 0, NULL, 0, NULL, NULL, 0, NULL), BAD);
    EXPECT(fp8_gemm_act_grad(A, 1, 0, B, 0, 0, D, 1, 8, 16, 32, F, 1, F, 1, 2, NULL, 1, NULL, NULL, 0, NULL, NULL, 0, NULL), BAD);
    EXPECT(fp8_gemm_act_grad(A, 1, 0, B, 0, 0, D, 1, 8, 16, 32, F, 1, F, 1, 2, Z, 1, F, S, 63, NULL, NULL, 0, NULL), BAD);
    EXPECT(fp8_gemm_act_grad(A, 1, 0, B, 0, 0, D, 1, 8, 16, 32, F, 1, F, 1, 2, D, 0, NULL, NULL, 0, NULL, NULL, 0, NULL), BAD);
    EXPECT(fp8_gemm_gated(A, 0, 0, B, 0, 1, D, 1, 8, 16, 32, F, 1, F, 16, 4, Z, 1, NULL, NULL, 0, NULL), BAD);
    EXPECT(fp8_gemm_gated(A, 0, 0, B, 0, 1, D, 1, 8, 16, 32, F, 1, F, 1, 4, D, 1, NULL, NULL, 0, NULL), BAD);
    EXPECT(fp8_gemm_gated_grad(A, 1, 0, B, 0, 0, D, 1, 8, 16, 32, F, 1, F, 2, 4, Z, 1, NULL, NULL, 0, NULL), BAD);
    EXPECT(fp8_gemm_gated_grad(A, 1, 0, B, 0, 0, D, 1, 8, 16, 32, F, 1, F, 1, 4, NULL, 1, NULL, NULL, 0, NULL), BAD);
    EXPECT(fp8_gemm_gated_grad(A, 1, 0, B, 0, 0, D, 1, 8, 16, 32, F, 1, F, 1, 4, D, 0, NULL, NULL, 0, NULL), BAD);
    EXPECT(fp8_gemm_gated_grad(A, 1, 0, B, 0, 0, D, 1, (int64_t)1 << 40, 1, (int64_t)1 << 40, F, 1, F, 1, 4, D, 0, NULL, NULL, 0, NULL), BAD);      /* byte counts beyond 2^63 */
}

static void workspaces(void)
{
    EXPECT(fp8_gemm_act_grad_workspace_size(33, 10), 80);
    EXPECT(fp8_gemm_act_grad_workspace_size(32, 10), 40);
    EXPECT(fp8_gemm_act_grad_workspace_size(1, 1), 4);
    EXPECT(fp8_gemm_act_grad_workspace_size(0, 10), 0);
    EXPECT(fp8_gemm_act_grad_workspace_size(INT64_MIN, INT64_MIN), 0);
    EXPECT(fp8_gemm_act_grad_workspace_size(INT64_MAX, 1) == (size_t)1 << 60, 1);
    EXPECT(fp8_gemm_act_grad_workspace_size((int64_t)1 << 40, (int64_t)1 << 18) == (size_t)1 << 55, 1);
    EXPECT(fp8_gemm_act_grad_workspace_size(INT64_MAX, INT64_MAX) == SIZE_MAX, 1);          /* more than a size_t holds */
    EXPECT(fp8_gemm_act_grad_workspace_size((int64_t)1 << 40, (int64_t)1 << 40) == SIZE_MAX, 1);
}

/* Nothing to compute: what is written without a product, and nothing else. */
static void empty(void)
{
    LAUNCHES(fp8_gemm_act(NULL, 0, 0, NULL, 0, 1, NULL, 1, 0, 16, 32, F, 0, F, 1, 2, NULL, 0, NULL, 0, NULL, 0, NULL, NULL, 0, NULL), FP8_OK, 0, 0);
    LAUNCHES(fp8_gemm_act(NULL, 0, 0, NULL, 0, 1, NULL, 1, 8, 0, 32, F, 1, F, 0, 2, NULL, 0, NULL, 0, NULL, 0, NULL, F, 0, NULL), FP8_OK, 1, 1);      /* the maximum */
    LAUNCHES(fp8_gemm_act_grad(NULL, 1, 0, NULL, 0, 0, NULL, 1, 0, 100, 32, F, 1, F, 1, 2, NULL, 1, F, NULL, 0, NULL, NULL, 0, NULL), FP8_OK, 1, 2);  /* the bias gradient */
    LAUNCHES(fp8_gemm_act_grad(NULL, 1, 0, NULL, 0, 0, NULL, 1, 0, 100, 32, F, 1, F, 1, 2, NULL, 1, F, NULL, 0, NULL, F, 0, NULL), FP8_OK, 2, 3);
    LAUNCHES(fp8_gemm_gated(NULL, 0, 0, NULL, 0, 1, NULL, 1, 0, 16, 32, F, 1, F, 1, 4, NULL, 1, NULL, NULL, 0, NULL), FP8_OK, 0, 0);
    LAUNCHES(fp8_gemm_gated_grad(NULL, 1, 0, NULL, 0, 0, NULL, 1, 8, 0, 32, F, 1, F, 1, 4, NULL, 1, NULL, NULL, 0, NULL), FP8_OK, 0, 0);
    LAUNCHES(fp8_gemm_act(NULL, 0, 0, NULL, 0, 1, D, 1, 8, 16, 0, F, 1, F, 1, 2, NULL, 0, NULL, 0, NULL, 0, NULL, NULL, 0, NULL), FP8_OK, 1, 1);      /* K = 0 */
}

/* Every product over shapes, storage orders, formats, alignments, flags and sides: one launch for it, one for the maximum where no other
 * carries it, one for the column sums.  What no grid holds is refused. */
static void products(void)
{
    for (int i = 0; i < 12000; ++i) {
        const int most = i % 10 == 0 ? 36 : 14;
        const int64_t M = draw_size(most), N = draw_size(most), K = draw_size(most);
        const uint64_t r = draw();
        const int tA = (int)(r & 1), tB = (int)(r >> 1 & 1), fA = (int)(r >> 2 & 1), fB = (int)(r >> 3 & 1), kind = (int)(r >> 4 & 3), flags = (int)(r >> 6 & 1);
        const int act = (int)((r >> 7) % 5), off = (int)(r >> 12 & 15) * (int)(r >> 16 & 1), amax = (int)(r >> 17 & 1), sums = (int)(r >> 18 & 1), dt = (int)(r >> 19 & 1);
        const int64_t nsA = r >> 20 & 1 ? M : 1;
        const int op = (int)(draw() % 4);
        float* const top = amax ? F + 64 : NULL;
        const float* const sD = kind >= FP8_OUT_E4M3 ? F + 32 : NULL;
        const int64_t cols = op == 2 ? 2 * N : N, nsB = r >> 21 & 1 ? cols : 1;
        const size_t need = sums ? fp8_gemm_act_grad_workspace_size(M, N) : 0;
        int got, most_launches = 1 + amax;
        recorded_launches = recorded_workgroups = 0;
        switch (op) {
            case 0: got = fp8_gemm_act(A + off, fA, tA, B, fB, tB, D, kind, M, N, K, F, nsA, F, nsB, act, S, dt, sums ? (void*)AT(7) : NULL, dt, amax ? Z : NULL, 1 - dt, sD, top, flags, NULL); break;
            case 1:
                got = fp8_gemm_act_grad(A + off, fA, tA, B, fB, tB, D, kind, M, N, K, F, nsA, F, nsB, act, Z, dt, sums ? F + 128 : NULL, S, need, sD, top, flags, NULL);
                most_launches += sums;
                break;
            case 2: got = fp8_gemm_gated(A + off, fA, tA, B, fB, tB, D, kind, M, N, K, F, nsA, F, nsB, act, sums ? Z : NULL, dt, sD, top, flags, NULL); break;
            default: got = fp8_gemm_gated_grad(A + off, fA, tA, B, fB, tB, D, kind, M, N, K, F, nsA, F, nsB, act, Z, dt, sD, top, flags, NULL); break;
        }
        /* (no output of fewer than 2^24 tiles of 64 x 64 is refused, nor one whose operands fit between the stand-ins' addresses) */
        const double tiles = ((double)M / 64 + 1) * ((double)cols / 64 + 1), apart = (double)((int64_t)1 << 43);
        const int long_operand = (double)M * (double)K > apart || (double)cols * (double)K > apart || (double)M * (double)cols * 8.0 > apart;
        const int fine = got == FP8_OK ? recorded_launches >= 1 && recorded_launches <= (unsigned long long)most_launches
                                       : got == BAD ? long_operand : tiles >= (double)(1 << 24) && (got == FP8_ERR_UNSUPPORTED || got == FP8_ERR_DEVICE);
        if (!fine) {
            printf("op %d of %lld x %lld x %lld, draw %llx: %d after %llu launches (%s)\n", op, (long long)M, (long long)N, (long long)K, (unsigned long long)r, got, recorded_launches,
                   fp8_last_error());
            ++failures;
        }
    }
}

/* Lists of tensors: none, one, empty ones among them, more than a launch holds, longer than 2^32 chunks together. */
static void gradients(void)
{
    enum { MOST = 1000 };
    static const void* x[MOST];
    static void* out[MOST];
    static size_t n[MOST];
    static int dtype[MOST];
    for (int i = 0; i < MOST; ++i) { x[i] = (const void*)(AT(8) + ((uintptr_t)i << 30)); out[i] = (void*)(AT(9) + ((uintptr_t)i << 30)); n[i] = 100; dtype[i] = i & 1; }
    EXPECT(fp8_grad_norm(-1, x, n, dtype, F, S, NULL), BAD);
    EXPECT(fp8_grad_norm(1, NULL, n, dtype, F, S, NULL), BAD);
    EXPECT(fp8_grad_norm(1, x, n, dtype, NULL, S, NULL), BAD);
    EXPECT(fp8_grad_norm(1, x, n, dtype, F, (char*)S + 4, NULL), BAD);
    EXPECT(fp8_grad_clip(1, x, n, dtype, NULL, F, -1.0f, NULL), BAD);
    EXPECT(fp8_grad_clip(1, x, n, dtype, NULL, NULL, 1.0f, NULL), BAD);
    LAUNCHES(fp8_grad_norm(0, NULL, NULL, NULL, F, S, NULL), FP8_OK, 1, 1);
    LAUNCHES(fp8_grad_clip(0, NULL, NULL, NULL, NULL, F, 1.0f, NULL), FP8_OK, 0, 0);
    LAUNCHES(fp8_grad_norm(1, x, n, dtype, F, S, NULL), FP8_OK, 1, 1);
    LAUNCHES(fp8_grad_norm(240, x, n, dtype, F, S, NULL), FP8_OK, 1, 240);
    LAUNCHES(fp8_grad_norm(241, x, n, dtype, F, S, NULL), FP8_OK, 2, 241);
    LAUNCHES(fp8_grad_norm(MOST, x, n, dtype, F, S, NULL), FP8_OK, 5, MOST);
    LAUNCHES(fp8_grad_clip(160, x, n, dtype, out, F, 1.0f, NULL), FP8_OK, 1, 160);
    LAUNCHES(fp8_grad_clip(161, x, n, dtype, out, F, 1.0f, NULL), FP8_OK, 2, 161);
    LAUNCHES(fp8_grad_clip(MOST, x, n, dtype, NULL, F, 1.0f, NULL), FP8_OK, 7, MOST);
    out[700] = (char*)x[700] + 2 * (700 & 1 ? 1 : 2);
    LAUNCHES(fp8_grad_clip(MOST, x, n, dtype, out, F, 1.0f, NULL), BAD, 0, 0);                      /* overlaps in part, the others are fine */
    out[700] = NULL;
    LAUNCHES(fp8_grad_clip(MOST, x, n, dtype, out, F, 1.0f, NULL), BAD, 0, 0);
    out[700] = (void*)x[700];
    LAUNCHES(fp8_grad_clip(MOST, x, n, dtype, out, F, 1.0f, NULL), FP8_OK, 7, MOST);
    for (int i = 0; i < MOST; ++i) { n[i] = i % 3 ? 0 : 16384 * 2 + 1; if (!n[i]) { x[i] = NULL; out[i] = NULL; } }
    LAUNCHES(fp8_grad_norm(MOST, x, n, dtype, F, S, NULL), FP8_OK, 2, 3 * 334);
    LAUNCHES(fp8_grad_clip(MOST, x, n, dtype, out, F, 1.0f, NULL), FP8_OK, 3, 3 * 334);
    for (int i = 0; i < MOST; ++i) n[i] = 0;
    LAUNCHES(fp8_grad_norm(MOST, x, n, dtype, F, S, NULL), FP8_OK, 1, 1);
    LAUNCHES(fp8_grad_clip(MOST, x, n, dtype, out, F, 1.0f, NULL), FP8_OK, 0, 0);
    for (int i = 0; i < 3; ++i) { x[i] = (const void*)AT(8 + i); n[i] = (size_t)1 << 45; dtype[i] = FP8_BF16; }     /* 2^31 chunks each: a launch of its own */
    LAUNCHES(fp8_grad_norm(3, x, n, dtype, F, S, NULL), FP8_OK, 3, 3 * 2048);
    LAUNCHES(fp8_grad_clip(3, x, n, dtype, NULL, F, 1.0f, NULL), FP8_OK, 3, 3 * 65536);
}

int main(void)
{
    refusals();
    workspaces();
    empty();
    products();
    gradients();
    if (failures) { printf("%d failure(s)\n", failures); return 1; }
    printf("ok\n");
    return 0;
}
