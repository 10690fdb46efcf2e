"""The feed-forward operators with weights of more than 2^32 bytes, where the halves of a gated block's weight lie 2^31 bytes apart and more:
the first and last outputs and those around the middle against 64 bits.  Tolerances as in test_gpu_ffn.py."""
import pytest
import torch

import paper_2209_05433_amd as fp8
import test_gpu_ffn as ffn
from test_gpu_ffn import BF16, E4M3, F32

pytestmark = pytest.mark.gpu


def weight(rows, cols, seed):
    """FP8 bytes of 2^-3 .. 2^3 either sign, drawn in pieces."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    b = torch.empty(rows, cols, dtype=torch.uint8, device="cuda")
    flat = b.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        n = min(1 << 28, flat.numel() - i)
        v = torch.randint(0, 96, (n,), generator=gen, dtype=torch.uint8, device="cuda")
        flat[i:i + n] = (v % 48 + 32) | (v // 48) * 128                      # exponents 4 .. 9 of bias 7, a sign
    return b


def columns(n):
    """Which outputs are looked at."""
    return torch.cat([torch.arange(64), torch.arange(n // 2 - 70, n // 2 + 70), torch.arange(n - 64, n)]).cuda()


def product(a, b):
    """Sums in 64 bits of FP8 bytes a [M, K] and b [n, K], with the bound."""
    a, b = a.view(torch.float8_e4m3fn).double(), b.view(torch.float8_e4m3fn).double()
    c = a @ b.t()
    return c, 2.0 ** -20 * (a.abs() @ b.abs().t()) + 2.0 ** -22 * c.abs()


@pytest.mark.parametrize("M,F,K", [(130, 200000, 16384), (130, 280000, 16384), (20, 280000, 16384), (3, 2048, 1 << 21)])
def test_gated(M, F, K):
    A, B, one = weight(M, K, 1), weight(2 * F, K, 2), torch.ones(1, device="cuda")
    H, GU = torch.empty(M, F, device="cuda"), torch.empty(M, 2 * F, device="cuda")
    fp8.fp8_gemm_gated(A, E4M3, False, B, E4M3, True, H, F32, one, one, ffn.ACTS["relu"], GU)
    at = columns(F)
    g, eg = product(A, B[at])
    u, eu = product(A, B[at + F])
    ffn.accept(GU[:, at], F32, g, eg, what="g")
    ffn.accept(GU[:, at + F], F32, u, eu, what="u")
    want = torch.relu(g) * u
    ffn.accept(H[:, at], F32, want, eg * (u.abs() + eu) + torch.relu(g) * eu + 2.0 ** -21 * want.abs(), what="H")


@pytest.mark.parametrize("M,N,K", [(300, 400000, 16384), (20, 400000, 16384), (3, 4096, 1 << 21), (40, 100001, 65536)])
def test_product_and_gradient(M, N, K):
    A, B, one = weight(M, K, 3), weight(N, K, 4), torch.ones(1, device="cuda")
    D = torch.empty(M, N, device="cuda")
    at = columns(N)
    c, E = product(A, B[at])
    fp8.fp8_gemm_act(A, E4M3, False, B, E4M3, True, D, F32, one, one, ffn.ACTS["relu"])
    ffn.accept(D[:, at], F32, torch.relu(c), E, what="D")
    Z = torch.randn(M, N, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").bfloat16()
    db = torch.empty(N, device="cuda")
    ws = torch.empty(fp8.fp8_gemm_act_grad_workspace_size(M, N), dtype=torch.uint8, device="cuda")
    fp8.fp8_gemm_act_grad(A, E4M3, False, B, E4M3, True, D, F32, one, one, ffn.ACTS["relu"], Z, db, ws)
    want = c * (Z[:, at] > 0)
    ffn.accept(D[:, at], F32, want, E, what="dZ")
    ffn.accept(db[at], F32, want.sum(0), E.sum(0) + M * 2.0 ** -24 * want.abs().sum(0), what="dbias")


@pytest.mark.parametrize("M,F,K", [(130, 65552, 40000), (20, 65544, 40000)])
def test_gated_with_a_weight_stored_in_out(M, F, K):
    A, B, one = weight(M, K, 6), weight(K, 2 * F, 7), torch.ones(1, device="cuda")
    H = torch.empty(M, F, dtype=torch.bfloat16, device="cuda")
    fp8.fp8_gemm_gated(A, E4M3, False, B, E4M3, False, H, BF16, one, one, ffn.ACTS["relu"])
    at = columns(F)
    g, eg = product(A, B[:, at].t().contiguous())
    u, eu = product(A, B[:, at + F].t().contiguous())
    want = torch.relu(g) * u
    ffn.accept(H[:, at], BF16, want, eg * (u.abs() + eu) + torch.relu(g) * eu + 2.0 ** -21 * want.abs(), what="H")
