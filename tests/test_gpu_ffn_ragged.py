"""The tiled form of the feed-forward operators where rows do not end on a lane's eight columns, and where the tensors beside the
product begin off 16 bytes while the operands do not: everything that test_gpu_ffn.py's sizes, multiples of 8 in that form, leave out."""
import pytest
import torch

import paper_2209_05433_amd as fp8
import test_gpu_ffn as ffn
from test_gpu_ffn import BF16, E5M2, F32, O43, O52

pytestmark = pytest.mark.gpu

TILED = ["tiled_256", "tiled_128", "tiled_both"]
# (a column short of and beyond a lane's eight, a wave's and a tile's columns; B stored N x K with K % 16 = 0: any N is the tiled kernel's)
SIZES = [(1, 3, 64), (130, 65, 272), (70, 131, 64), (257, 257, 128), (300, 1001, 272), (513, 1003, 16)]
F, H = torch.float32, torch.bfloat16


@pytest.fixture(params=[0, 1, 3], ids=lambda k: "beside_%d" % k)
def beside(request, monkeypatch):
    """Elements by which bias, residual, z and g | u begin off 16 bytes; outputs begin there by the case's shift."""
    k = request.param
    if k:
        def off(t, D):
            if t is None or t is D or t.numel() == 0:
                return t
            buf = torch.full((t.numel() + 16,), float("nan"), dtype=t.dtype, device="cuda")
            buf[k:k + t.numel()] = t.flatten()
            return buf[k:k + t.numel()].view(t.shape)

        def wrap(call, *which):
            def moved(*args):
                args = list(args)
                for i in which:
                    args[i] = off(args[i], args[6])
                return call(*args)
            return moved
        monkeypatch.setattr(fp8, "fp8_gemm_act", wrap(fp8.fp8_gemm_act, 11, 12))
        monkeypatch.setattr(fp8, "fp8_gemm_act_grad", wrap(fp8.fp8_gemm_act_grad, 11))
        monkeypatch.setattr(fp8, "fp8_gemm_gated_grad", wrap(fp8.fp8_gemm_gated_grad, 11))
    return k


def case(k, *size, **more):
    """Aligned operands, outputs that begin k elements off."""
    c = ffn.Case(*size, **more)
    c.shift = k
    return c


@pytest.mark.parametrize("name", TILED)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_products(M, N, K, name, beside):
    for i, (kind, act, bias, residual, z) in enumerate([(BF16, "gelu", H, None, H), (F32, "silu", F, F, None), (O43, "relu", None, H, F), (O52, "none", H, F, H)]):
        c = case(beside, M, N, K, per_row=i == 1, factors="column" if i in (1, 2) else "one", flags=i % 2, seed=50 + i)
        ffn.run_act(c, act, kind, bias=bias, residual=residual, z=z, name=name)


@pytest.mark.parametrize("name", TILED)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_gradients(M, N, K, name, beside):
    for i, (kind, act, z) in enumerate([(O52, "gelu", H), (F32, "silu", F), (BF16, "gelu_tanh", F), (O43, "none", H)]):
        c = case(beside, M, N, K, fA=E5M2, per_row=i == 1, factors="column" if i in (1, 2) else "one", flags=i % 2, seed=60 + i)
        ffn.run_act_grad(c, act, kind, z=z, name=name)


@pytest.mark.parametrize("name", TILED)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_gated(M, N, K, name, beside):
    for i, (kind, act, gu) in enumerate([(BF16, "silu", H), (F32, "gelu", None), (O43, "gelu_tanh", F), (O52, "relu", H)]):
        c = case(beside, M, N, K, wide=True, per_row=i == 1, factors=["one", "column", "pair", "one"][i], flags=i % 2, seed=70 + i)
        ffn.run_gated(c, act, kind, gu=gu, name=name)


@pytest.mark.parametrize("name", TILED)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_gated_gradients(M, N, K, name, beside):
    for i, (kind, act, gu) in enumerate([(O52, "silu", H), (F32, "gelu", F), (BF16, "gelu_tanh", F), (O43, "none", H)]):
        c = case(beside, M, N, K, fA=E5M2, per_row=i == 1, factors="column" if i in (1, 2) else "one", flags=i % 2, seed=80 + i)
        ffn.run_gated_grad(c, act, kind, gu=gu, name=name)


@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("name", TILED)
@pytest.mark.parametrize("M,N,K", [(130, 65, 272), (300, 1001, 64), (300, 1000, 64)])
def test_in_place(M, N, K, name, shift):
    for kind, dtype in ((BF16, H), (F32, F)):
        ffn.run_act(case(shift, M, N, K, seed=90), "gelu", kind, bias=H, residual=dtype, z=F, in_place=True, name=name)
        ffn.run_act_grad(case(shift, M, N, K, fA=E5M2, seed=91), "silu", kind, z=dtype, in_place=True, name=name)
        ffn.run_gated_grad(case(shift, M, N, K, fA=E5M2, seed=92), "gelu", kind, gu=dtype, in_place=True, name=name)
