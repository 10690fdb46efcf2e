"""What the feed-forward operators refuse, on the host: nothing is launched, no pointer dereferenced."""
import ctypes

import pytest

import paper_2209_05433_amd as fp8

L = fp8.lib()
A, B, D, F, S, Z = 1 << 20, 1 << 24, 1 << 36, 1 << 40, 1 << 41, 1 << 42            # made-up aligned addresses, far apart
BAD, UNSUPPORTED = fp8.FP8_ERR_INVALID_ARG, fp8.FP8_ERR_UNSUPPORTED
M, N, K = 8, 16, 32


def act(**k):
    a = dict(A=A, fmtA=0, transA=0, B=B, fmtB=0, transB=1, D=D, out_kind=1, M=M, N=N, K=K, sA=F, nsA=1, sB=F, nsB=1, act=2, bias=None, bias_dtype=0, residual=None,
             residual_dtype=0, Z=None, Z_dtype=0, sD=None, amax=None, flags=0, stream=None)
    assert set(k) <= set(a)
    a.update(k)
    return L.fp8_gemm_act(*a.values())


def act_grad(**k):
    a = dict(A=A, fmtA=1, transA=0, B=B, fmtB=0, transB=0, D=D, out_kind=1, M=M, N=N, K=K, sA=F, nsA=1, sB=F, nsB=1, act=2, Z=Z, Z_dtype=1, dbias=None, workspace=None,
             workspace_bytes=0, sD=None, amax=None, flags=0, stream=None)
    assert set(k) <= set(a)
    a.update(k)
    return L.fp8_gemm_act_grad(*a.values())


def gated(grad=False, **k):
    a = dict(A=A, fmtA=0, transA=0, B=B, fmtB=0, transB=1, D=D, out_kind=1, M=M, N=N, K=K, sA=F, nsA=1, sB=F, nsB=1, act=4, GU=Z, GU_dtype=1, sD=None, amax=None, flags=0,
             stream=None)
    assert set(k) <= set(a)
    a.update(k)
    return (L.fp8_gemm_gated_grad if grad else L.fp8_gemm_gated)(*a.values())


EACH = [act, act_grad, gated, lambda **k: gated(True, **k)]


@pytest.mark.parametrize("wrong,word", [
    (dict(fmtA=2), "fp8_format_t"), (dict(fmtB=-1), "fp8_format_t"), (dict(transA=2), "transA"), (dict(transB=-1), "transA"), (dict(out_kind=4), "fp8_out_t"),
    (dict(act=5), "fp8_act_t"), (dict(act=-1), "fp8_act_t"), (dict(M=-1), "negative"), (dict(N=-1), "negative"), (dict(K=-1), "negative"), (dict(sA=None), "NULL"),
    (dict(sB=None), "NULL"), (dict(nsA=2), "nsA"), (dict(nsB=5), "nsB"), (dict(sA=F + 2), "misaligned"), (dict(sB=F + 1), "misaligned"), (dict(amax=F + 2), "misaligned"),
    (dict(sD=F), "FP8 outputs"), (dict(D=None), "NULL"), (dict(A=None), "A or B"), (dict(B=None), "A or B"), (dict(D=D + 1), "aligned"), (dict(flags=2), "flag"),
    (dict(out_kind=0, D=D + 2), "aligned")])
def test_what_all_products_refuse(wrong, word):
    for call in EACH:
        assert call(**wrong) == BAD and word in fp8.fp8_last_error(), fp8.fp8_last_error()


def test_sizes_beyond_what_bytes_can_be_counted():
    for call in EACH:
        assert call(M=(1 << 40) + 1) == UNSUPPORTED
        assert call(M=1 << 35, N=1 << 35) == UNSUPPORTED


def test_tensors_beside_the_product():
    assert act(bias=S + 1, bias_dtype=1) == BAD and act(bias=S + 2, bias_dtype=0) == BAD and act(bias=S, bias_dtype=2) == BAD
    assert act(residual=S, residual_dtype=-1) == BAD and act(residual=S + 1, residual_dtype=1) == BAD
    assert act(Z=Z, Z_dtype=7) == BAD and act(Z=Z + 2, Z_dtype=0) == BAD
    # overlaps: the residual may be D, of one type; Z may be nothing else
    assert act(residual=D, residual_dtype=0) == BAD and act(residual=D + 2, residual_dtype=1) == BAD
    assert act(residual=D + M * N * 2 - 2, residual_dtype=1) == BAD and act(residual=D - M * N * 2 + 2, residual_dtype=1) == BAD
    assert act(Z=D, Z_dtype=1) == BAD and act(Z=A, Z_dtype=1) == BAD and act(Z=B + N * K - 4, Z_dtype=1) == BAD and act(Z=S, Z_dtype=1, residual=S, residual_dtype=1) == BAD
    assert act_grad(Z=None) == BAD and act_grad(Z_dtype=2) == BAD and act_grad(Z=D, Z_dtype=0) == BAD and act_grad(Z=D + 2) == BAD
    assert gated(GU=D) == BAD and gated(GU=A) == BAD and gated(GU=B + 2 * N * K - 2) == BAD and gated(GU_dtype=3) == BAD
    assert gated(True, GU=None) == BAD and gated(True, GU=D, GU_dtype=0) == BAD and gated(True, GU=D + 4) == BAD and gated(True, GU=Z + 1) == BAD
    assert gated(nsB=N) == BAD and "2F" in fp8.fp8_last_error()                    # one per column of op(B) means 2F of them


def test_workspace_of_the_bias_gradient():
    assert fp8.fp8_gemm_act_grad_workspace_size(33, 10) == 2 * 10 * 4
    assert fp8.fp8_gemm_act_grad_workspace_size(0, 10) == fp8.fp8_gemm_act_grad_workspace_size(5, 0) == fp8.fp8_gemm_act_grad_workspace_size(-1, 5) == 0
    need = fp8.fp8_gemm_act_grad_workspace_size(M, N)
    assert act_grad(dbias=F, workspace=None) == BAD and act_grad(dbias=F, workspace=S, workspace_bytes=need - 1) == BAD
    assert act_grad(dbias=F, workspace=S + 2, workspace_bytes=need) == BAD and act_grad(dbias=F + 1, workspace=S, workspace_bytes=need) == BAD


def test_gradient_lists():
    vp, sz, i = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    lists = lambda x, n, d: ((vp * len(x))(*x), (sz * len(n))(*n), (i * len(d))(*d))
    norm = lambda x, n, d, out=F, ws=S, count=None: L.fp8_grad_norm(len(x) if count is None else count, *lists(x, n, d), out, ws, None)
    clip = lambda x, n, d, o=None, cell=F, most=1.0: L.fp8_grad_clip(len(x), *lists(x, n, d), o and (vp * len(o))(*o), cell, most, None)
    assert norm([A], [4], [0], count=-1) == BAD and L.fp8_grad_norm(1, None, None, None, F, S, None) == BAD
    for call in (norm, clip):
        assert call([A], [4], [2]) == BAD and call([None], [4], [0]) == BAD and call([A + 2], [4], [0]) == BAD and call([A, A + 1], [4, 4], [0, 1]) == BAD
        assert call([A], [1 << 46], [0]) == UNSUPPORTED
    assert norm([A], [4], [0], out=None) == BAD and norm([A], [4], [0], out=F + 2) == BAD and norm([A], [4], [0], ws=None) == BAD and norm([A], [4], [0], ws=S + 4) == BAD
    assert clip([A], [4], [0], cell=None) == BAD and clip([A], [4], [0], cell=F + 2) == BAD
    assert clip([A], [4], [0], most=-1.0) == BAD and clip([A], [4], [0], most=float("nan")) == BAD
    assert clip([A], [4], [0], o=[None]) == BAD and clip([A], [4], [0], o=[D + 2]) == BAD and clip([A], [4], [0], o=[A + 4]) == BAD
