// The loss over a vocabulary: a row's pairs joined (gemm_loss.hpp; gfx950).
#include "gemm_loss.hpp"

namespace fp8mm {
namespace {

// Workgroups of 256: ROWS rows, 256 / ROWS threads each, which take the row's pairs in turn; their parts meet in LDS in a fixed order.  In 64 bits,
// which cost nothing here.  Neighbouring threads take neighbouring rows, as the pairs lie in memory.
// Few rows: a launch and a chain of loads (one of 50257 columns 4.6 us, 1001 of 6283 4.8); 4096 and 8192 rows of 50257 columns read 13 and 26 MB of pairs in 6.9 and
// 11.1 us, a hundredth of their products.
template <int ROWS>
__global__ __launch_bounds__(256) void loss_join_kernel(LossArgs o, int64_t blocks, int64_t M, int64_t N, float* __restrict__ loss, float* __restrict__ lse)
{
    constexpr int PARTS = 256 / ROWS;
    __shared__ float refs[PARTS][ROWS];
    __shared__ double sums[PARTS][ROWS];
    const int r = threadIdx.x % ROWS, part = threadIdx.x / ROWS;
    const int64_t row = (int64_t)blockIdx.x * ROWS + r;
    const LossPair* pairs = (const LossPair*)o.partials + (row < M ? row : M - 1);
    float ref = -3.4028234663852886e38f;
    double sum = 0.0;
    // (the part of the smaller reference is brought to the larger one; what lies more than 2^126 below adds nothing)
    auto add = [&](float other, double s) __attribute__((always_inline)) {
        const float top = __builtin_fmaxf(ref, other);
        sum = sum * (double)__builtin_amdgcn_exp2f(ref - top) + s * (double)__builtin_amdgcn_exp2f(other - top);
        ref = top;
    };
    int64_t b = part;
    for (; b + 3 * PARTS < blocks; b += 4 * PARTS) {
        LossPair p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = pairs[(b + i * PARTS) * M];
#pragma unroll
        for (int i = 0; i < 4; ++i) add(p[i].ref, (double)p[i].sum);
    }
    for (; b < blocks; b += PARTS) {
        const LossPair p = pairs[b * M];
        add(p.ref, (double)p.sum);
    }
    refs[part][r] = ref;
    sums[part][r] = sum;
    __syncthreads();
    for (int half = PARTS / 2; half >= 1; half >>= 1) {
        if (part < half) {
            add(refs[part + half][r], sums[part + half][r]);
            refs[part][r] = ref;
            sums[part][r] = sum;
        }
        __syncthreads();
    }
    if (part != 0 || row >= M) return;
    const float l = (float)(((double)ref + log2(sum)) * 0.69314718055994530942);
    lse[row] = l;
    const int64_t y = label_column(o, row);
    float v = l;
    if (o.z_weight != 0.0f) v = __builtin_fmaf(o.z_weight * l, l, v);
    if (y >= 0 && y < N) v -= loss_targets(o, M, N)[row];
    loss[row] = y == -1 ? 0.0f : v;
}

}  // namespace

int launch_loss_join(const LossArgs& o, int64_t blocks, int64_t M, int64_t N, float* loss, float* lse, hipStream_t stream)
{
    // as many rows a workgroup as leave a workgroup for every compute unit; all threads at a single row where there are few
    const int rows = M >= 256 * 32 ? 32 : M >= 256 * 4 ? 8 : 1;
    const int64_t grid = (M + rows - 1) / rows;
    auto kern = rows == 32 ? loss_join_kernel<32> : rows == 8 ? loss_join_kernel<8> : loss_join_kernel<1>;
    enqueue(kern, dim3((unsigned)grid), dim3(256), 0, stream, o, blocks, M, N, loss, lse);
    return check_launch("loss over a vocabulary (join)");
}

}  // namespace fp8mm
