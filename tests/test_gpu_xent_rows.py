"""The loss over a vocabulary around the numbers of rows at which its second launch changes (one, eight or 32 rows a workgroup: from 1024 and from 8192 on), and its gradient where
exponentials vanish.  Tolerances: test_gpu_xent.py."""
import math

import pytest
import torch

import paper_2209_05433_amd as fp8
from test_gpu_xent import BF16, F32, FORMS, Problem, form

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["chosen", "small_32x32", "tiled_256", "tiled_128"])
@pytest.mark.parametrize("M", [1023, 1024, 1027, 1031, 8191, 8192, 8201])
@pytest.mark.parametrize("N", [1, 33, 3001])
def test_rows_of_a_workgroup(M, N, name):
    """(3001 columns: 94 blocks of 32, more than the 32 threads of a row; 1: fewer)"""
    with form(name):
        Problem(M, N, 32, seed=M + N, first=N).check_loss(z_weight=1e-2)


@pytest.mark.parametrize("M", [1027, 8201])
def test_rows_of_infinities_among_others(M):
    """Rows whose logits are all -infinity, that hold an infinity, or a NaN, beside ordinary ones in the same workgroup."""
    N, inf = 700, math.inf
    p = Problem(M, N, 16, fa=fp8.FP8_E5M2, fb=fp8.FP8_E4M3, seed=3)
    a = p.A.view(torch.float8_e5m2).float().clone()
    w = p.B.view(torch.float8_e4m3fn).float()
    a[:, 0] = 0.0
    w[:, 0] = 1.0
    kinds = {3: -inf, 8: inf, 13: math.nan, M - 1: -inf, M - 2: inf}
    for row, value in kinds.items():
        a[row, 0] = value
    p.set(a.to(torch.float8_e5m2), w.to(torch.float8_e4m3fn))
    p.labels[[8, 3]] = 5
    loss, lse = p.loss()
    assert float(lse[3]) == float(lse[M - 1]) == -inf and float(lse[8]) == float(lse[M - 2]) == inf and math.isnan(float(lse[13]))
    rest = torch.ones(M, dtype=torch.bool, device="cuda")
    rest[list(kinds)] = False
    # (0 times an infinity nowhere: a row's own element is the infinite one)
    sizes = p.sizes.clone()
    p.sizes = torch.where(rest[:, None], sizes, torch.zeros_like(sizes))
    want, tol, want_lse, tol_lse = p.expected_loss()
    assert bool(((lse.double() - want_lse).abs() <= tol_lse)[rest].all()) and bool(((loss.double() - want).abs() <= tol)[rest].all())


@pytest.mark.parametrize("name", FORMS)
@pytest.mark.parametrize("dloss", [1.0, 2.0 ** 60])
def test_exponentials_that_vanish(name, dloss):
    """Logits of up to 110 below their row's sum: the exponential is within 2^-22 (|z| + |lse| + 4) of itself or within 2^-126 of it, y accordingly by dloss (1 + 2 z_weight lse) more."""
    w = 1e-2
    with form(name):
        p = Problem(70, 600, 64, seed=4, spread=1.0)
        lse = (torch.logsumexp(p.z, 1) + torch.linspace(60.0, 105.0, 70, device="cuda").double()).float()
        for out in (F32, BF16):
            D = p.gradient(out, lse, torch.full((1,), dloss, device="cuda"), w).double()
            l = lse.double()[:, None]
            scale = dloss * (1 + 2 * w * l)
            e = torch.exp(p.z - l)
            hot = (torch.arange(p.N, device="cuda") + p.first)[None, :] == p.labels[:, None]
            y = torch.where((p.labels < 0)[:, None], 0, scale * e - dloss * hot)
            tol = scale * (e * torch.expm1(p.bound + 2.0 ** -22 * (p.z.abs() + l.abs() + 4)) + 2.0 ** -126) + 2.0 ** -23 * dloss * hot
            half = y.abs() * (2.0 ** -8 if out == BF16 else 2.0 ** -24) + 2.0 ** -134
            assert bool(((D - y).abs() <= 1.01 * tol + half).all()), ((D - y).abs() / (tol + half)).max()
            vanish = (e < 2.0 ** -127) & ~hot
            assert int(vanish.sum()) > 1000 and bool((D[vanish].abs() <= 1.01 * (scale * 2.0 ** -126).expand_as(D)[vanish]).all())
