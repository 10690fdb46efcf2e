"""FP8_GEMM_MFMA8 on the products with an operator behind them: the FP8 instructions where the tiled kernel's shapes allow them, and
fp8_gemm's arithmetic and bound everywhere else (include/fp8mm.h, fp8_gemm_mfma8).

The operands' magnitudes are spread over 17 binades, so that a run of 8 products on the FP8 instructions loses bits: by up to 2^-13 of its
largest product, many times the 2^-20 of the sum of magnitudes that fp8_gemm grants.  Tolerances as in test_gpu_ffn.py, for calls
without the flag."""
import math

import pytest
import torch

import paper_2209_05433_amd as fp8
import test_gpu_ffn as ffn
from test_gpu_ffn import BF16, E4M3, E5M2, F32

pytestmark = pytest.mark.gpu


def spread(c, wide=False):
    """The case with operands of magnitudes 2^-8.5 .. 2^8.5 and the bound of fp8_gemm, flag or not."""
    cols = 2 * c.N if wide else c.N

    def draw(stored, rows, cols, fmt, trans):
        shape = (cols, rows) if trans else (rows, cols)
        e = 17.0 * torch.rand(shape, generator=c.gen, device="cuda") - 8.5
        sign = 1.0 - 2.0 * torch.randint(0, 2, shape, generator=c.gen, device="cuda")
        q = (sign * torch.exp2(e)).to(ffn.TORCH8[fmt])
        stored.copy_(q.view(torch.uint8))
        q = q.double()
        return q.t().contiguous() if trans else q
    a = draw(c.A, c.M, c.K, c.fA, c.tA)
    b = draw(c.B, c.K, cols, c.fB, c.tB)
    rms = math.sqrt(2.0 ** 17 / (17 * 2 * math.log(2)))
    scale = rms * math.sqrt(math.sqrt(c.K))
    c.sA.mul_(scale / c.sA.mean())
    c.sB.mul_(scale / c.sB.mean())
    per = c.sA.double().reshape(-1, 1) * c.sB.double().reshape(1, -1)
    c.c = (a @ b) / per
    c.E = 2.0 ** -20 * ((a.abs() @ b.abs()) / per) + 2.0 ** -22 * c.c.abs()
    return c


RUNS = {
    "act": lambda c, name: ffn.run_act(c, "relu", F32, bias=torch.float32, name=name),
    "act_grad": lambda c, name: ffn.run_act_grad(c, "relu", F32, z=torch.float32, name=name)[0],
    "gated": lambda c, name: ffn.run_gated(c, "relu", F32, gu=torch.float32, name=name),
    "gated_grad": lambda c, name: ffn.run_gated_grad(c, "relu", F32, gu=torch.float32, name=name),
}

# outside the tiled kernel: odd K; a B stored K x N whose rows begin off 16 bytes; operands that begin off 16 bytes; K = 100 with neither
# operand contiguous along it (the tiled kernel takes that in fp8_gemm's arithmetic), the last with a weight in E5M2 too
OUTSIDE = [dict(M=90, N=200, K=333), dict(M=300, N=1000, K=512, tB=False), dict(M=64, N=128, K=256, shift=3), dict(M=272, N=144, K=100, tA=True, tB=False),
           dict(M=528, N=272, K=333, tA=True, tB=False, fB=E5M2)]


@pytest.mark.parametrize("name", ["chosen", "small_32x32", "small_32x64", "small_64x64", "tiled_256"])
@pytest.mark.parametrize("op", list(RUNS))
@pytest.mark.parametrize("shape", OUTSIDE, ids=lambda s: "x".join(str(s[k]) for k in "MNK") + ("_off" if "shift" in s else ""))
def test_shapes_outside_the_tiled_kernel_are_computed_as_without_the_flag(op, shape, name):
    got = []
    for flags in (fp8.FP8_GEMM_MFMA8, 0):
        c = spread(ffn.Case(flags=flags, seed=41, wide=op == "gated", **shape), op == "gated")
        got.append(RUNS[op](c, name))
    assert torch.equal(got[0], got[1])
