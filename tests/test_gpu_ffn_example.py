"""The feed-forward operators as a program uses them: examples/ffn_step.py against autograd in 32 bits, and its training steps."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("ffn_step", os.path.join(ROOT, "examples", "ffn_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def near(a, b):
    """Cosine of two tensors and the ratio of their norms."""
    a, b = a.double().flatten(), b.double().flatten()
    return float(a @ b / a.norm() / b.norm()), float(a.norm() / b.norm())


@pytest.mark.parametrize("kind", ["gated", "mlp"])
@pytest.mark.parametrize("tokens,width,inner", [(512, 256, 768), (300, 200, 520)])
def test_block_against_autograd(kind, tokens, width, inner):
    """Outputs and every gradient against 32-bit autograd of the same block.  FP8 rounds operands to 2^-4 (E4M3) and 2^-3 (E5M2, and it
    enters a gradient once or twice): errors of a few per cent of independent terms, cosines above 0.99."""
    ex = example()
    block = ex.Block(kind, tokens, width, inner, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(tokens, width, generator=gen, device="cuda").to(torch.bfloat16)
    dy = (1e-4 * torch.randn(tokens, width, generator=gen, device="cuda")).to(torch.bfloat16)
    block.b1.normal_(std=0.1, generator=gen)
    block.b2.normal_(std=0.1, generator=gen)
    y = block.forward(x)
    dx = block.backward(dy)
    leaves = [t.float().clone().requires_grad_(True) for t in (x, block.W1, block.W2, block.b1, block.b2)]
    xr, w1, w2, b1, b2 = leaves
    if kind == "gated":
        g, u = (xr @ w1.t()).chunk(2, 1)
        ref = xr + (torch.nn.functional.silu(g) * u) @ w2.t()
    else:
        ref = xr + torch.nn.functional.gelu(xr @ w1.t() + b1) @ w2.t() + b2
    ref.backward(dy.float())
    pairs = [(y, ref), (dx, xr.grad), (block.dW1, w1.grad), (block.dW2, w2.grad)] + ([(block.db1, b1.grad)] if kind == "mlp" else [])
    for a, b in pairs:
        cosine, ratio = near(a, b)
        assert cosine > 0.99 and 0.95 < ratio < 1.05, (cosine, ratio)


@pytest.mark.parametrize("kind", ["gated", "mlp"])
def test_training_steps(kind):
    runs = list(example().train(kind, 1024, 256, 768, 12))
    losses = [l for l, _ in runs]
    assert all(b < a for a, b in zip(losses, losses[1:])) and losses[-1] < 0.9 * losses[0], losses
    assert all(n > 0 and n == n for _, n in runs)


def test_a_token():
    ex = example()
    for kind in ("gated", "mlp"):
        one, many = ex.Block(kind, 1, 256, 768, seed=5), ex.Block(kind, 40, 256, 768, seed=5)
        x = torch.randn(40, 256, generator=torch.Generator(device="cuda").manual_seed(6), device="cuda").to(torch.bfloat16)
        a, b = one.forward(x[:1].contiguous(), train=False), many.forward(x)
        cosine, ratio = near(a, b[:1])
        assert cosine > 0.995 and 0.97 < ratio < 1.03          # (the factors of the casts differ)
