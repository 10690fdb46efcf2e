"""Memory that the gradient of the loss writes and that is an argument otherwise too: refused on the host, nothing is launched."""
import pytest

import paper_2209_05433_amd as fp8
from test_step_refusals import A, B, BAD, D, F, K, M, N, S, Z, grad

# (the gradient of test_step_refusals: D of M x N bytes at D, factors at F, dloss at F + 64, labels at S, lse at Z)


@pytest.mark.parametrize("wrong", [
    dict(D=F - M * N + 1), dict(D=F), dict(sA=D + 4), dict(sB=D + M * N - 4), dict(sA=D + M * N - 4, nsA=M), dict(sA=D - 4 * M + 4, nsA=M), dict(sB=D - 4 * N + 4, nsB=N), dict(sD=D + 8), dict(amax=D),
    dict(amax=D + M * N - 4), dict(out_kind=0, amax=D + 4 * M * N - 4), dict(amax=A), dict(amax=A + M * K - 4), dict(amax=B + 4), dict(amax=S), dict(amax=S + 8 * M - 4), dict(amax=Z + 4 * M - 4)])
def test_the_gradient(wrong):
    assert grad(**wrong) == BAD and "overlap" in fp8.fp8_last_error(), fp8.fp8_last_error()


def test_an_output_of_nothing_overlaps_nothing():
    assert grad(N=0, D=S + 8) == fp8.FP8_OK and grad(M=0, ndloss=1, D=F + 64) == fp8.FP8_OK
