"""AdamW to the last bit, and where its numbers leave the ordinary range."""
import pytest
import torch

import paper_2209_05433_amd as fp8

pytestmark = pytest.mark.gpu


def cells(value, dtype=torch.float32):
    return torch.full((1,), value, dtype=dtype, device="cuda")


def test_the_clipping_factor():
    """beta1 = 0 and gradients of 1: m' is the factor itself.  max_norm times the rounded reciprocal, which is what torch makes of a number over a tensor."""
    g = torch.ones(5, device="cuda")
    norms = torch.exp(torch.linspace(-9.0, 9.0, 301, device="cuda"))
    for most in (0.3, 1.0, 1e-3):
        got = []
        for norm in norms.split(1):
            p, m, v = (torch.zeros(5, device="cuda") for _ in range(3))
            fp8.fp8_adamw([p], [g], [m], [v], cells(1, torch.int64), cells(0.0), beta1=0.0, norm=norm, max_norm=most)
            got.append(m[:1])
        assert torch.equal(torch.cat(got), (most / (norms + 1e-6)).clamp(max=1.0))
