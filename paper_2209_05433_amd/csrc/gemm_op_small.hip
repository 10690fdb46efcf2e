// Products with an operator behind them on small output tiles, any shape and any alignment, for gfx950 (MI355X).
//
// The K loop is that of the plain product's kernel of small tiles (gemm_small.hip: tiles of 32 x 32, 32 x 64 and 64 x 64 columns of op(B), the
// waves of a workgroup share K, chunks fetched as they lie in memory and turned into fragments in the wave's own piece of LDS; the same
// instructions and the same order of sums).  What is different is how it ends: the waves' sums, added in wave order, go through op_row
// four columns at a time.  With two columns of op(B) for each output (the gated block) the tile's first 32 columns are the gate's and the
// other 32 the second projection's of the same 32 outputs: a thread adds up both before it combines them, and no sum goes through memory.
// Column sums (the bias gradient) are added over the tile's rows in a fixed order and leave as one row of partial sums per row of tiles.
//
// This file is compiled once per pair of storage orders: -DFP8MM_LAYOUT.
#include "gemm_small_tile.hpp"
#include "gemm_op.hpp"

#include <atomic>
#include <type_traits>

namespace fp8mm {
namespace {

// Operand B of the gated block: two blocks, the 32 columns of op(B) from t0 on and the 32 from F + t0 on (F >= 16 where they are
// contiguous in memory).
template <bool KC, int S>
struct PairOperand : Operand<KC, 2, S> {
    typedef Operand<KC, 2, S> Base;
    using Base::PIECES; using Base::CK; using Base::LPR; using Base::RPL;
    int64_t F;

    __device__ __forceinline__ void setup(const uint8_t* p, int64_t F_, int64_t K_, int64_t t0, int l)
    {
        F = F_; this->ext = 2 * F; this->K = K_;
        const int row = l / LPR;
        if (KC) {
            const int64_t r = t0 + row < F ? t0 + row : F - 1;
            this->base = p + r * this->K + 16 * (l % LPR);
            this->last = F - 1 - r < 32 ? (int)(F - 1 - r) : 32;
            this->shift = 0; this->edge = false;
        } else {
            this->edge = t0 + 32 > F;
            const int64_t own = t0 + 16 * (l & 1), col = own + 16 <= F ? own : F - 16;
            this->base = p + col + (l % LPR >= 2 ? F : 0);
            this->shift = own - col < 15 ? (int)(own - col) : 15;
            this->last = row;
        }
    }
    __device__ __forceinline__ const uint8_t* row_of(int q) const          // KC: the lane's row of load q
    {
        const int r = q * RPL % 32;
        return this->base + (int64_t)(r < this->last ? r : this->last) * this->K + (q * RPL >= 32 ? F * this->K : 0);
    }
    __device__ __forceinline__ void fetch(u32x4 (&x)[PIECES], int64_t c) const
    {
#pragma unroll
        for (int q = 0; q < PIECES; ++q)
            x[q] = KC ? *(const u32x4_any*)(row_of(q) + c * CK) : *(const u32x4_any*)(this->base + (c * CK + q * RPL + this->last) * this->ext);
    }
    __device__ __forceinline__ void fetch_guarded(u32x4 (&x)[PIECES], int64_t c, int l) const
    {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
            if (KC) {
                const int at = 16 * (l % LPR);
                x[q] = load_guarded(row_of(q) - at, c * CK + at, this->K);
            } else {
                const int64_t k = c * CK + q * RPL + this->last;
                x[q] = k >= this->K ? (u32x4){0u, 0u, 0u, 0u} : *(const u32x4_any*)(this->base + k * this->ext);
            }
        }
    }
};

// Tile of 32 RM rows and 32 RN columns of op(B), NW waves, D chunks in flight per wave.  PAIR: the gated block (RN = 2).
template <int FMT_A, int FMT_B, int ACC, bool A_KC, bool B_KC, int RM, int RN, int S, int NW, int D, bool PAIR>
__global__ __launch_bounds__(64 * NW) void gemm_op_small_kernel(const uint8_t* __restrict__ A, const uint8_t* __restrict__ B, void* C,
                                                                int64_t M, int64_t N, int64_t K, OpArgs o)
{
    typedef Operand<A_KC, RM, S> OpA;
    typedef typename std::conditional<PAIR, PairOperand<B_KC, S>, Operand<B_KC, RN, S>>::type OpB;
    constexpr int CK = S * SK, WIDTH = 32 * RN / (PAIR ? 2 : 1);          // output columns of the tile
    constexpr int PER_WAVE = small_lds_per_wave<A_KC, B_KC, RM, RN, S>();
    constexpr int RED = 32 * RM * RED_PITCH * 4;          // bytes of a wave's sums
    static_assert(PER_WAVE - RED >= 32 * (RM + RN) * 8, "the reciprocals of the factors lie behind the first wave's sums");
    static_assert(NW * 32 * RN * 4 + NW * 4 <= NW * PER_WAVE - RED && NW >= 2, "column sums and maxima behind the first wave's block");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];       // NW * PER_WAVE
    const int tid = threadIdx.x, l = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);

    // tiles down the rows of D first; every XCD gets one contiguous run (see gemm_small.hip)
    const int64_t tiles_m = (M + 32 * RM - 1) / (32 * RM), total = gridDim.x;
    const int64_t x = blockIdx.x % 8, idx = blockIdx.x / 8, share = total / 8, rem = total % 8;
    const int64_t p = x * share + (x < rem ? x : rem) + idx;
    const int64_t tm = p % tiles_m, m0 = tm * (32 * RM), n0 = (p / tiles_m) * WIDTH;

    // the factors that the thread will take the reciprocals of, loaded while the products run
    const bool uniform = !o.a_per_row && o.b_factors == B_ONE;
    constexpr int FACTORS = (RM + RN + 2 * NW - 1) / (2 * NW);            // per thread
    float factor[FACTORS];
#pragma unroll
    for (int f = 0; f < FACTORS; ++f) {
        const int t = tid + f * 64 * NW, c = t - 32 * RM;
        factor[f] = 1.0f;
        if (o.a_per_row && t < 32 * RM) factor[f] = o.sA_dev[m0 + t < M ? m0 + t : M - 1];
        if (o.b_factors != B_ONE && c >= 0 && c < 32 * RN) {
            const bool up = PAIR && c >= 32;
            const int64_t n = n0 + (PAIR ? c & 31 : c), col = n < N ? n : N - 1;
            factor[f] = o.sB_dev[o.b_factors == B_COLUMN ? col + (up ? N : 0) : up ? 1 : 0];
        }
    }

    OpA a; OpB b;
    a.setup(A, M, K, m0, l);
    b.setup(B, N, K, n0, l);
    uint8_t* slab_a = lds + w * PER_WAVE;
    uint8_t* slab_b = slab_a + OpA::SLAB;

    v16f acc[RN][RM];
#pragma unroll
    for (int i = 0; i < RN; ++i)
#pragma unroll
        for (int j = 0; j < RM; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

    auto multiply = [&](const u32x4 (&xa)[OpA::PIECES], const u32x4 (&xb)[OpB::PIECES]) __attribute__((always_inline)) {
        a.store(xa, slab_a, l);
        b.store(xb, slab_b, l);
#pragma unroll
        for (int sub = 0; sub < S; ++sub) {
            v8i fa[RM], fb[RN];
            a.fragments(slab_a, sub, l, fa);
            b.fragments(slab_b, sub, l, fb);
            if (ACC == ACC_FP8) {
#pragma unroll
                for (int i = 0; i < RN; ++i)
#pragma unroll
                    for (int j = 0; j < RM; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[i], fa[j], acc[i][j], FMT_B, FMT_A, 0, 0, 0, 0);
            } else {
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    v8h ha[RM], hb[RN];
#pragma unroll
                    for (int j = 0; j < RM; ++j) ha[j] = widen8<FMT_A>(fa[j][2 * s], fa[j][2 * s + 1]);
#pragma unroll
                    for (int i = 0; i < RN; ++i) hb[i] = widen8<FMT_B>(fb[i][2 * s], fb[i][2 * s + 1]);
#pragma unroll
                    for (int i = 0; i < RN; ++i)
#pragma unroll
                        for (int j = 0; j < RM; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(hb[i], ha[j], acc[i][j], 0, 0, 0);
                }
            }
        }
    };

    // chunks inside K without tests (a load for every step: the last ones repeat the wave's last chunk), then the others
    const int64_t chunks = (K + CK - 1) / CK;
    const int64_t plain = (A_KC || M >= 16) && (B_KC || N >= 16) ? K / CK : 0;
    const int64_t mine = plain > w ? (plain - w + NW - 1) / NW : 0;      // of this wave
    if (mine > 0) {
        u32x4 xa[D][OpA::PIECES], xb[D][OpB::PIECES];
        auto fetch = [&](int d, int64_t i) __attribute__((always_inline)) {
            const int64_t c = w + NW * (i < mine ? i : mine - 1);
            a.fetch(xa[d], c);
            b.fetch(xb[d], c);
        };
#pragma unroll
        for (int d = 0; d < D; ++d) fetch(d, d);
        int64_t i = 0;
        for (; i + D <= mine; i += D)
#pragma unroll
            for (int d = 0; d < D; ++d) {
                multiply(xa[d], xb[d]);
                fetch(d, i + d + D);
            }
#pragma unroll
        for (int d = 0; d < D - 1; ++d)
            if (i + d < mine) multiply(xa[d], xb[d]);
    }
    for (int64_t c = plain + (w + NW - plain % NW) % NW; c < chunks; c += NW) {
        u32x4 xa[OpA::PIECES], xb[OpB::PIECES];
        a.fetch_guarded(xa, c, l);
        b.fetch_guarded(xb, c, l);
        multiply(xa, xb);
    }

    // The waves' sums meet in LDS, 32 columns at a time.  The reciprocals of factors per row or column in 64 bits, as in the plain kernel.
    const double a_all = o.a_per_row ? 1.0 : (double)o.sA_dev[0], b_all = o.b_factors != B_ONE ? 1.0 : (double)o.sB_dev[0];
    const double r_all = 1.0 / (a_all * b_all);
    const float sD = o.out_kind >= OUT_E4M3 ? scale_value(o.sD_dev, 1.0f) : 1.0f;
    double* row_factors = (double*)(lds + RED);
    double* col_factors = row_factors + 32 * RM;
    constexpr int TRIPS = (32 * RM * 8 + 64 * NW - 1) / (64 * NW);       // rows that a thread takes four columns of
    float first[PAIR ? TRIPS : 1][4];
    float column[RN][4];                                  // sums over the thread's rows
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < RN; ++i) {
        __syncthreads();                                  // the slabs, or the block before, are done with
        if (i == 0 && !uniform) {
#pragma unroll
            for (int f = 0; f < FACTORS; ++f)
                if (tid + f * 64 * NW < 32 * (RM + RN)) *LDS_PTR(double, row_factors + tid + f * 64 * NW) = 1.0 / factor[f];
        }
        float* mine_red = (float*)(lds + w * PER_WAVE);
#pragma unroll
        for (int j = 0; j < RM; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *LDS_PTR(v4f, mine_red + (32 * j + (l & 31)) * RED_PITCH + 8 * q + 4 * (l >> 5)) =
                    (v4f){acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        __syncthreads();
        const int64_t gn = n0 + (PAIR ? 0 : 32 * i) + 4 * (tid & 7);
        const int left = gn < N ? (N - gn < 4 ? (int)(N - gn) : 4) : 0;
        float bias[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (!PAIR && o.bias && left > 0) load_row<4>(o.bias, o.bias_dtype, gn, left, bias);
#pragma unroll
        for (int e = 0; e < 4; ++e) column[i][e] = 0.0f;
#pragma unroll
        for (int trip = 0; trip < TRIPS; ++trip) {
            const int u = tid + trip * 64 * NW;
            const int64_t gm = m0 + (u >> 3);
            if (u >= 32 * RM * 8 || gm >= M || left <= 0) continue;
            const float* red = (const float*)lds + (u >> 3) * RED_PITCH + 4 * (u & 7);
            v4f s = *LDS_PTR(v4f, red);
#pragma unroll
            for (int v = 1; v < NW; ++v) s += *LDS_PTR(v4f, red + v * (PER_WAVE / 4));
            float y[4], z[4], factors[4] = {(float)r_all, (float)r_all, (float)r_all, (float)r_all};
            if (!uniform) {
                const double ra = r_all * *LDS_PTR(double, row_factors + (u >> 3));
#pragma unroll
                for (int e = 0; e < 4; ++e) factors[e] = (float)(ra * *LDS_PTR(double, col_factors + 32 * i + 4 * (u & 7) + e));
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = s[e] * factors[e];
            if (PAIR && i == 0) {
#pragma unroll
                for (int e = 0; e < 4; ++e) first[PAIR ? trip : 0][e] = y[e];
                continue;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                z[e] = PAIR ? y[e] : 0.0f;
                if (PAIR) y[e] = first[PAIR ? trip : 0][e];
            }
            top = max(top, op_row<4, PAIR>(o, C, N, gm, gn, left, y, z, bias, sD));
#pragma unroll
            for (int e = 0; e < 4; ++e) column[i][e] += y[e];
        }
    }
    if (!PAIR && o.sums) {
        // over the wave's rows, then over the waves, in their order; behind the first wave's sums and the factors, which have been read
        float* cells = (float*)(lds + RED);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RN; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float s = column[i][e];
#pragma unroll
                for (int d = 8; d <= 32; d <<= 1) s += __shfl_xor(s, d, 64);
                if (l < 8) *LDS_PTR(float, cells + w * 32 * RN + 32 * i + 4 * l + e) = s;
            }
        __syncthreads();
        if (tid < 32 * RN && n0 + tid < N) {
            float s = 0.0f;
            for (int v = 0; v < NW; ++v) s += *LDS_PTR(float, cells + v * 32 * RN + tid);
            o.sums[tm * N + n0 + tid] = s;
        }
    }
    if (o.amax_out) {
        // one atomic per workgroup
        unsigned* cells = (unsigned*)(lds + RED + NW * 32 * RN * 4);
        __syncthreads();
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, d, 64));
        if (l == 0) *LDS_PTR(unsigned, cells + w) = top;
        __syncthreads();
        if (w == 0) op_commit_top(o, l < NW ? *LDS_PTR(unsigned, cells + l) : 0u);
    }
}

template <int FA, int FB, int ACC, int RM, int RN, int S, int NW, int D, bool PAIR>
int launch_form(const GemmArgs& g, const OpArgs& o)
{
    constexpr bool A_KC = (FP8MM_LAYOUT & 2) == 0, B_KC = (FP8MM_LAYOUT & 1) != 0;
    constexpr int LDS = NW * small_lds_per_wave<A_KC, B_KC, RM, RN, S>(), WIDTH = 32 * RN / (PAIR ? 2 : 1);
    auto kern = gemm_op_small_kernel<FA, FB, ACC, A_KC, B_KC, RM, RN, S, NW, D, PAIR>;
    if (LDS > 65536) {
        // more dynamic LDS than the default limit: raised once per device
        static std::atomic<unsigned long long> attr_set{0ull};
        if (int e = raise_lds_limit((const void*)kern, LDS, attr_set)) return e;
    }
    const int64_t tiles = ((g.M + 32 * RM - 1) / (32 * RM)) * ((g.N + WIDTH - 1) / WIDTH);
    enqueue(kern, dim3((unsigned)tiles), dim3(64 * NW), LDS, g.stream, g.A, g.B, g.C, g.M, g.N, g.K, o);
    return check_launch("gemm with an operator (small tiles)");
}

template <int FA, int FB, int ACC, bool PAIR>
int launch_acc(const GemmArgs& g, const OpArgs& o, int form)
{
    constexpr bool A_KC = (FP8MM_LAYOUT & 2) == 0, B_KC = (FP8MM_LAYOUT & 1) != 0;
    switch (form) {
        case SMALL_32x32:                                 // (the gated block: 32 outputs of a row are 64 columns of op(B))
            return launch_form<FA, FB, ACC, 1, PAIR ? 2 : 1, 2, 8, PAIR ? 1 : 2, PAIR>(g, o);
        case SMALL_32x64: return launch_form<FA, FB, ACC, 1, 2, 2, 4, 2, PAIR>(g, o);
    }
    if constexpr (A_KC && B_KC) {
        if (form == SMALL_64x64_LINES8) return launch_form<FA, FB, ACC, 2, 2, 2, 8, 1, PAIR>(g, o);
        if (form == SMALL_64x64_LINES4) return launch_form<FA, FB, ACC, 2, 2, 2, 4, 1, PAIR>(g, o);
    }
    return launch_form<FA, FB, ACC, 2, 2, 1, 4, 1, PAIR>(g, o);
}

template <int FA, int FB>
int launch_formats(const GemmArgs& g, const OpArgs& o, int form)
{
    if (op_pair_in(o.op)) return g.acc == ACC_FP8 ? launch_acc<FA, FB, ACC_FP8, true>(g, o, form) : launch_acc<FA, FB, ACC_F16, true>(g, o, form);
    return g.acc == ACC_FP8 ? launch_acc<FA, FB, ACC_FP8, false>(g, o, form) : launch_acc<FA, FB, ACC_F16, false>(g, o, form);
}

}  // namespace

#if !defined(FP8MM_LAYOUT)
#error "compile with -DFP8MM_LAYOUT=0..3 (2 * transA + transB)"
#endif

int FP8MM_OP_SMALL_NAME(FP8MM_LAYOUT)(const GemmArgs& g, const OpArgs& o, int form)
{
    if (g.fmtA == FP8_E4M3)
        return g.fmtB == FP8_E4M3 ? launch_formats<FP8_E4M3, FP8_E4M3>(g, o, form) : launch_formats<FP8_E4M3, FP8_E5M2>(g, o, form);
    return g.fmtB == FP8_E4M3 ? launch_formats<FP8_E5M2, FP8_E4M3>(g, o, form) : launch_formats<FP8_E5M2, FP8_E5M2>(g, o, form);
}

}  // namespace fp8mm
