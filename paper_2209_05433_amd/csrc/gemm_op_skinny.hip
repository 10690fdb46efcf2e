// Products of a few rows (the tokens of a decoding step) with an operator behind them, for gfx950 (MI355X).
//
//   up to 16 rows of A (M x K) times a weight stored [out, in] (B: N x K, or 2 N x K for the gated block), see gemm_op.hpp
//
// Every byte of the weight is used once per row and read once: bound by the stream of the weight where it is long, and by the chain launch - loads -
// sums - outputs where it is short.  A workgroup takes 16 outputs (16 rows of B; of the gated block those 16 and the same 16 of the second
// projection), its waves share K, 256 bytes of each row a trip.  The loads go straight into the layout of v_mfma_f32_16x16x32_f16: lane (r, g) =
// (l % 16, l / 16) holds 16 bytes of row r from 64 i + 16 g on, so that four lanes ask for 64 bytes side by side and nothing passes
// through LDS; the low and the high 8 of the 16 bytes go to two instructions, for A's rows and B's alike (a product is a sum over K in any order).
// The bytes are widened exactly to fp16 and summed in 32 bits; the waves' sums meet in LDS and are added in wave order.  A trip's
// loads are in flight while the trip before is multiplied.
// For outputs of few columns, where tiles of 32 x 32 (which read 32 rows of A for every 32 of B and turn both through LDS) leave compute units idle
// (see op_skinny_takes).
#include "gemm_op.hpp"

namespace fp8mm {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int SKINNY_M = 16, SKINNY_N = 16, PIECES = 4;         // 64-byte pieces of a row in a trip
constexpr int PITCH = SKINNY_N + 4;                             // floats between two rows of a wave's sums

template <int FMT_A, int FMT_B, int NW, bool PAIR>
__global__ __launch_bounds__(64 * NW) void gemm_op_skinny_kernel(const uint8_t* __restrict__ A, const uint8_t* __restrict__ B, void* D, int M, int64_t N, int64_t K, OpArgs o)
{
    constexpr int P = PAIR ? 2 : 1;
    __shared__ __attribute__((aligned(16))) float red[NW][P][SKINNY_M][PITCH];
    const int tid = threadIdx.x, l = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = l & 15, g = l >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * SKINNY_N;
    const uint8_t* a_row = A + (int64_t)(r < M ? r : M - 1) * K;                    // (rows beyond M or N: products that nobody looks at)
    const int64_t b_index = n0 + r < N ? n0 + r : N - 1;
    const uint8_t* b_row[P];
#pragma unroll
    for (int p = 0; p < P; ++p) b_row[p] = B + (b_index + p * N) * K;

    struct Trip { u32x4 a[PIECES], b[P][PIECES]; };
    // Beyond the end of K A's piece is zero, and B's the row's last one, where no infinity (0 x inf) can be: a NaN there is in the sum anyway.
    auto fetch = [&](Trip& t, int64_t trip) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int64_t k = trip * (64 * PIECES) + 64 * i + 16 * g, at = k < K ? k : K - 16;
            t.a[i] = *(const u32x4*)(a_row + at);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                t.b[p][i] = *(const u32x4*)(b_row[p] + at);
                if (FMT_B == FP8_E5M2 && k >= K) t.b[p][i] = (u32x4){0u, 0u, 0u, 0u};
            }
            if (k >= K) t.a[i] = (u32x4){0u, 0u, 0u, 0u};
        }
    };
    v4f acc[P][2] = {};
    auto multiply = [&](const Trip& t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const v8h a = widen8<FMT_A>((int)t.a[i][2 * h], (int)t.a[i][2 * h + 1]);
#pragma unroll
                for (int p = 0; p < P; ++p)
                    acc[p][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8<FMT_B>((int)t.b[p][i][2 * h], (int)t.b[p][i][2 * h + 1]), a, acc[p][h], 0, 0, 0);
            }
    };
    const int64_t trips = (K + 64 * PIECES - 1) / (64 * PIECES);
    if (w < trips) {
        Trip now, next;
        fetch(now, w);
        int64_t t = w + NW;
        for (; t < trips; t += NW) {
            fetch(next, t);
            multiply(now);
            now = next;
        }
        multiply(now);
    }
    // lane (r, g) has columns 4 g .. 4 g + 3 of row r
#pragma unroll
    for (int p = 0; p < P; ++p) *(v4f*)&red[w][p][r][4 * g] = acc[p][0] + acc[p][1];
    __syncthreads();
    if (w != 0) return;
    // four columns of a row a thread
    const int row = l >> 2, q = l & 3;
    const int64_t col = n0 + 4 * q;
    const int left = col < N ? (int)(N - col < 4 ? N - col : 4) : 0;
    float y[4] = {0.0f, 0.0f, 0.0f, 0.0f}, u[4] = {0.0f, 0.0f, 0.0f, 0.0f}, bias[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    unsigned top = 0;
    if (row < M && left > 0) {
        const double a = 1.0 / (double)o.sA_dev[o.a_per_row ? row : 0];
        if (o.bias) load_row<4>(o.bias, o.bias_dtype, col, left, bias);
        v4f s[P];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            s[p] = *(const v4f*)&red[0][p][row][4 * q];
            for (int v = 1; v < NW; ++v) s[p] += *(const v4f*)&red[v][p][row][4 * q];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t c = e < left ? col + e : col;
            y[e] = s[0][e] * (float)(a * op_column_factor(o, N, c, false));
            u[e] = PAIR ? s[P - 1][e] * (float)(a * op_column_factor(o, N, c, true)) : 0.0f;
        }
        const float sD = o.out_kind >= OUT_E4M3 ? scale_value(o.sD_dev, 1.0f) : 1.0f;
        top = op_row<4, PAIR>(o, D, N, row, col, left, y, u, bias, sD);
    }
    if (!PAIR && o.sums) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float s = row < M ? y[e] : 0.0f;
#pragma unroll
            for (int d = 4; d <= 32; d <<= 1) s += __shfl_xor(s, d, 64);
            if (row == 0 && e < left) o.sums[col + e] = s;
        }
    }
    if (o.amax_out) op_commit_top(o, top);
}

template <int FA, int FB>
void enqueue_skinny(const GemmArgs& g, const OpArgs& o, unsigned tiles)
{
    if (op_pair_in(o.op)) enqueue(gemm_op_skinny_kernel<FA, FB, 8, true>, dim3(tiles), dim3(512), 0, g.stream, g.A, g.B, g.C, (int)g.M, g.N, g.K, o);
    else enqueue(gemm_op_skinny_kernel<FA, FB, 8, false>, dim3(tiles), dim3(512), 0, g.stream, g.A, g.B, g.C, (int)g.M, g.N, g.K, o);
}

}  // namespace

// Up to 4096 columns of op(B): half as many columns a workgroup are twice as many workgroups.  Beyond, the wider tiles fill the chip and read A less
// often (us, one row, here / tiles of 32 x 32 or 32 x 64, the better; K behind the x: 768 x 768 3.8 / 4.1, 2048 x 2048 4.0 / 5.0, 2048 x 6144 6.2 / 8.0,
// 512 x 8192 7.1 / 9.2, 4096 x 4096 6.5 / 6.6, 6144 x 2048 5.7 / 5.7, 8192 x 4096 9.6 / 8.4, 6144 x 8192 13.2 / 10.9; gated 1000 x 1008 3.4 / 5.5,
// 2048 x 2048 5.0 / 6.4, 2048 x 6144 9.2 / 11.6, 4096 x 4096 11.3 / 10.0; 16 rows: 2048 x 6144 7.9 / 8.3, 4096 x 4096 7.1 / 6.8; an empty kernel takes 3.8 - 4.5 among others).
bool op_skinny_takes(const GemmArgs& g, bool pair)
{
    return g.M <= SKINNY_M && !g.transA && g.transB && g.K >= 16 && g.K % 16 == 0 && (((uintptr_t)g.A | (uintptr_t)g.B) & 15) == 0 && (pair ? 2 : 1) * g.N <= 4096;
}

int launch_op_skinny(const GemmArgs& g, const OpArgs& o)
{
    const unsigned tiles = (unsigned)((g.N + SKINNY_N - 1) / SKINNY_N);
    if (g.fmtA == FP8_E4M3) {
        if (g.fmtB == FP8_E4M3) enqueue_skinny<FP8_E4M3, FP8_E4M3>(g, o, tiles);
        else enqueue_skinny<FP8_E4M3, FP8_E5M2>(g, o, tiles);
    } else {
        if (g.fmtB == FP8_E4M3) enqueue_skinny<FP8_E5M2, FP8_E4M3>(g, o, tiles);
        else enqueue_skinny<FP8_E5M2, FP8_E5M2>(g, o, tiles);
    }
    return check_launch("gemm with an operator (few rows)");
}

}  // namespace fp8mm
