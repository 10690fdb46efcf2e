/* Host-side exercise of the loss over a vocabulary, its gradient and AdamW, for a build of the library with AddressSanitizer and
 * UndefinedBehaviorSanitizer on the host code (tests/test_step_sanitizers.py): their argument checks, workspace sizes, choice of kernels over a seeded
 * sweep of shapes up to 2^36, and the lists of tensors that go into launches.  Launches are recorded and run nothing (tests/hip_recording_stub.c).
 * Exit status 0 and "ok" on stdout if every call returned what it should. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
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
#define AT(k) ((uintptr_t)(k) << 44)
#define A ((const uint8_t*)AT(1))
#define B ((const uint8_t*)AT(2))
#define D ((void*)AT(3))
#define F ((float*)AT(4))
#define Y ((const int64_t*)AT(5))
#define L ((float*)AT(6))
#define W ((void*)AT(7))

static uint64_t seed = 54321;
static uint64_t draw(void) { seed = seed * 6364136223846793005ull + 1442695040888963407ull; return seed >> 24; }
static int64_t draw_size(int most_bits)
{
    const int bits = (int)(draw() % (uint64_t)(most_bits + 1));
    const int64_t v = (int64_t)(((uint64_t)1 << bits) + (draw() & (((uint64_t)1 << bits) - 1)));
    switch (draw() % 4) { case 0: return v; case 1: return (v + 15) / 16 * 16; case 2: return (v + 255) / 256 * 256; default: return v > 3 ? v - 1 : v; }
}

static void workspaces(void)
{
    EXPECT(fp8_gemm_xent_workspace_size(33, 10), 33 * 16);
    EXPECT(fp8_gemm_xent_workspace_size(1, 0), 8);
    EXPECT(fp8_gemm_xent_workspace_size(0, 10), 0);
    EXPECT(fp8_gemm_xent_workspace_size(1, -1), 0);
    EXPECT(fp8_gemm_xent_workspace_size(INT64_MIN, INT64_MIN), 0);
    EXPECT(fp8_gemm_xent_workspace_size(1, INT64_MAX) == 8 * (((size_t)1 << 58) + 1), 1);
    EXPECT(fp8_gemm_xent_workspace_size(INT64_MAX, INT64_MAX) == SIZE_MAX, 1);
    EXPECT(fp8_gemm_xent_workspace_size((int64_t)1 << 40, (int64_t)1 << 40) == SIZE_MAX, 1);
}

/* Nothing to compute: what is written without a product, and nothing else. */
static void empty(void)
{
    LAUNCHES(fp8_gemm_xent(NULL, 0, 0, NULL, 0, 1, 0, 16, 32, F, 1, F, 1, NULL, 0, 0, NULL, NULL, NULL, 0, 0, NULL), FP8_OK, 0, 0);
    LAUNCHES(fp8_gemm_xent(NULL, 0, 0, NULL, 0, 1, 5, 0, 32, F, 1, F, 1, Y, 0, 0, L, L + 64, W, 40, 0, NULL), FP8_OK, 1, 5);              /* rows of nothing */
    LAUNCHES(fp8_gemm_xent(NULL, 0, 0, NULL, 0, 1, 5, 100, 0, F, 1, F, 1, Y, 0, 0, L, L + 64, W, 1000, 0, NULL), FP8_OK, 2, 2 + 5);       /* K = 0 */
    LAUNCHES(fp8_gemm_xent_grad(NULL, 0, 0, NULL, 0, 1, NULL, 1, 0, 16, 32, F, 1, F, 1, NULL, 0, 0, NULL, NULL, 1, NULL, NULL, 0, NULL), FP8_OK, 0, 0);
    LAUNCHES(fp8_gemm_xent_grad(NULL, 0, 0, NULL, 0, 1, NULL, 1, 5, 0, 32, F, 1, F, 1, Y, 0, 0, L, L, 1, NULL, F, 0, NULL), FP8_OK, 1, 1);        /* the maximum */
}

/* Both products over shapes, storage orders, formats, alignments and flags: one launch for the product, one for the join or the maximum.  What no grid holds is
 * refused. */
static void products(void)
{
    for (int i = 0; i < 12000; ++i) {
        const int most = i % 10 == 0 ? 36 : 14;
        const int64_t M = draw_size(most), N = draw_size(most), K = draw_size(most);
        const uint64_t r = draw();
        const int tA = (int)(r & 1), tB = (int)(r >> 1 & 1), fA = (int)(r >> 2 & r >> 16 & 1), fB = (int)(r >> 3 & r >> 17 & 1), kind = (int)(r >> 4 & 3), flags = (int)(r >> 6 & 1);
        const int off = (int)(r >> 12 & 15) * (int)(r >> 18 & 1), amax = (int)(r >> 19 & 1), grad = (int)(r >> 20 & 1);
        const int64_t nsA = r >> 21 & 1 ? M : 1, nsB = r >> 22 & 1 ? N : 1, nd = r >> 23 & 1 ? M : 1;
        const float* const sD = kind >= FP8_OUT_E4M3 ? F + 32 : NULL;
        int got;
        recorded_launches = recorded_workgroups = 0;
        if (grad) got = fp8_gemm_xent_grad(A + off, fA, tA, B, fB, tB, D, kind, M, N, K, F, nsA, F, nsB, Y, (int64_t)(r >> 24), 1e-4f, L, F, nd, sD, amax ? F + 64 : NULL, flags, NULL);
        else got = fp8_gemm_xent(A + off, fA, tA, B, fB, tB, M, N, K, F, nsA, F, nsB, Y, (int64_t)(r >> 24), 0.0f, L, (float*)AT(8), (void*)AT(9), SIZE_MAX, flags, NULL);
        const double tiles = ((double)M / 32 + 1) * ((double)N / 32 + 1), apart = (double)((int64_t)1 << 44);
        const int long_operand = (double)M * (double)K > apart || (double)N * (double)K > apart || (double)M * (double)N * 4.0 > apart;
        const int fine = got == FP8_OK ? recorded_launches == (unsigned long long)(grad ? 1 + amax : 2)
                                       : got == BAD ? long_operand : tiles >= (double)(1 << 22) && (got == FP8_ERR_UNSUPPORTED || got == FP8_ERR_DEVICE);
        if (!fine) {
            printf("%s of %lld x %lld x %lld, draw %llx: %d after %llu launches (%s)\n", grad ? "gradient" : "loss", (long long)M, (long long)N, (long long)K, (unsigned long long)r, got,
                   recorded_launches, fp8_last_error());
            ++failures;
        }
    }
}

/* Lists of tensors: none, one, empty ones among them, more than a launch holds, longer than 2^32 chunks together. */
static void adamw(void)
{
    enum { MOST = 300 };
    static void *p[MOST], *m[MOST], *v[MOST];
    static const void* g[MOST];
    static uint8_t* q[MOST];
    static float *ms[MOST], *vs[MOST], decay[MOST];
    static size_t n[MOST];
    static int pt[MOST], gt[MOST];
    for (int i = 0; i < MOST; ++i) {
        const uintptr_t at = (uintptr_t)i << 30;
        p[i] = (void*)(AT(10) + at); g[i] = (const void*)(AT(11) + at); m[i] = (void*)(AT(12) + at); v[i] = (void*)(AT(13) + at);
        q[i] = i & 1 ? (uint8_t*)(AT(14) + at) : NULL; ms[i] = (float*)(AT(15) + at); vs[i] = (float*)(AT(16) + at);
        n[i] = 100; pt[i] = i & 1; gt[i] = i >> 1 & 1; decay[i] = 0.1f;
    }
#define STEP(count, kind, q_, amax, flags) \
    fp8_adamw(count, p, pt, g, gt, n, m, v, kind, ms, vs, 1, decay, F, Y, 0.9, 0.999, 1e-8f, F, 1.0f, q_, 0, F + 64, amax, flags, NULL)
    EXPECT(STEP(-1, 0, NULL, NULL, 0), BAD);
    EXPECT(STEP(1, 2, NULL, NULL, 0), BAD);
    EXPECT(STEP(1, 0, NULL, NULL, 2), BAD);
    LAUNCHES(STEP(0, 0, q, F, 0), FP8_OK, 0, 0);
    LAUNCHES(fp8_adamw(0, NULL, NULL, NULL, NULL, NULL, NULL, NULL, 1, NULL, NULL, 1, NULL, F, Y, 0.9, 0.999, 1e-8f, NULL, NAN, NULL, 7, NULL, NULL, 0, NULL), FP8_OK, 0, 0);
    for (int kind = 0; kind < 2; ++kind) {
        LAUNCHES(STEP(1, kind, NULL, NULL, 0), FP8_OK, 1, 1);
        LAUNCHES(STEP(50, kind, q, NULL, 1), FP8_OK, 1, 50);
        LAUNCHES(STEP(51, kind, q, F, 1), FP8_OK, 3, 1 + 51);
        LAUNCHES(STEP(MOST, kind, q, NULL, 0), FP8_OK, 6, MOST);
    }
    p[200] = (char*)p[7] + 4 * (pt[7] ? 1 : 2);
    pt[200] = 1;
    LAUNCHES(STEP(MOST, 0, NULL, NULL, 0), BAD, 0, 0);              /* two of the weights overlap in part */
    p[200] = (char*)p[7] + 400;
    LAUNCHES(STEP(MOST, 0, NULL, NULL, 0), FP8_OK, 6, MOST);        /* one behind the other */
    decay[299] = NAN;
    LAUNCHES(STEP(MOST, 0, NULL, NULL, 0), BAD, 0, 0);
    decay[299] = 0.0f;
    for (int i = 0; i < MOST; ++i) { n[i] = i % 3 ? 0 : 4096 * 2 + 1; if (!n[i]) { p[i] = m[i] = v[i] = NULL; g[i] = NULL; q[i] = NULL; ms[i] = vs[i] = NULL; } }
    LAUNCHES(STEP(MOST, 1, q, NULL, 0), FP8_OK, 2, 3 * 100);
    for (int i = 0; i < MOST; ++i) n[i] = 0;
    LAUNCHES(STEP(MOST, 1, q, F, 0), FP8_OK, 1, 1);                 /* the maxima */
    for (int i = 0; i < 3; ++i) {                                   /* 2^29 chunks each; of 2^31 a launch of its own; more is refused */
        p[i] = (void*)AT(20 + i); g[i] = (const void*)AT(30 + i); m[i] = (void*)AT(40 + i); v[i] = (void*)AT(50 + i); ms[i] = (float*)AT(60 + i); vs[i] = (float*)AT(70 + i);
        n[i] = (size_t)1 << 41; pt[i] = gt[i] = FP8_BF16;
    }
    LAUNCHES(STEP(3, 1, NULL, NULL, 0), FP8_OK, 1, 65536);
    for (int i = 0; i < 3; ++i) n[i] = (size_t)1 << 43;
    LAUNCHES(STEP(3, 1, NULL, NULL, 0), FP8_OK, 3, 3 * 65536);
    n[1] += 1;
    LAUNCHES(STEP(3, 1, NULL, NULL, 0), FP8_ERR_UNSUPPORTED, 0, 0);
}

int main(void)
{
    workspaces();
    empty();
    products();
    adamw();
    if (failures) { printf("%d failure(s)\n", failures); return 1; }
    printf("ok\n");
    return 0;
}
