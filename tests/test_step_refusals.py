"""What the loss over a vocabulary, its gradient and AdamW refuse, on the host: nothing is launched, no pointer dereferenced."""
import ctypes
import math

import pytest

import paper_2209_05433_amd as fp8

L = fp8.lib()
A, B, D, F, S, Z, W = 1 << 20, 1 << 24, 1 << 36, 1 << 40, 1 << 41, 1 << 42, 1 << 43         # made-up aligned addresses, far apart
BAD, UNSUPPORTED = fp8.FP8_ERR_INVALID_ARG, fp8.FP8_ERR_UNSUPPORTED
M, N, K = 8, 16, 32
vp = ctypes.c_void_p


def xent(**k):
    a = dict(A=A, fmtA=0, transA=0, B=B, fmtB=0, transB=1, M=M, N=N, K=K, sA=F, nsA=1, sB=F, nsB=1, labels=S, first=0, z_weight=0.0, loss=Z, lse=Z + 4096, workspace=W,
             workspace_bytes=1 << 30, flags=0, stream=None)
    assert set(k) <= set(a)
    a.update(k)
    return L.fp8_gemm_xent(*a.values())


def grad(**k):
    a = dict(A=A, fmtA=0, transA=0, B=B, fmtB=0, transB=1, D=D, out_kind=3, M=M, N=N, K=K, sA=F, nsA=1, sB=F, nsB=1, labels=S, first=0, z_weight=0.0, lse=Z, dloss=F + 64,
             ndloss=1, sD=None, amax=None, flags=0, stream=None)
    assert set(k) <= set(a)
    a.update(k)
    return L.fp8_gemm_xent_grad(*a.values())


@pytest.mark.parametrize("wrong,word", [
    (dict(fmtA=2), "fp8_format_t"), (dict(fmtB=-1), "fp8_format_t"), (dict(transA=2), "transA"), (dict(transB=-1), "transA"), (dict(M=-1), "negative"), (dict(N=-1), "negative"),
    (dict(K=-1), "negative"), (dict(sA=None), "NULL"), (dict(sB=None), "NULL"), (dict(nsA=2), "nsA"), (dict(nsB=5), "nsB"), (dict(sA=F + 2), "misaligned"),
    (dict(A=None), "A or B"), (dict(B=None), "A or B"), (dict(flags=2), "flag"), (dict(labels=None), "labels"), (dict(labels=S + 4), "labels"), (dict(first=-1), "first"),
    (dict(z_weight=-1e-4), "z_weight"), (dict(z_weight=math.inf), "z_weight"), (dict(z_weight=math.nan), "z_weight")])
def test_what_both_products_refuse(wrong, word):
    for call in (xent, grad):
        assert call(**wrong) == BAD and word in fp8.fp8_last_error(), fp8.fp8_last_error()


@pytest.mark.parametrize("wrong,word", [
    (dict(loss=None), "loss"), (dict(loss=Z + 2), "loss"), (dict(lse=None), "NULL"), (dict(lse=Z + 2), "aligned"), (dict(workspace=None), "workspace"),
    (dict(workspace=W + 4), "workspace"), (dict(workspace_bytes=8 * M * 2 - 1), "workspace"), (dict(lse=Z), "overlap"), (dict(lse=Z + 4 * (M - 1)), "overlap"),
    (dict(workspace=Z), "overlap"), (dict(labels=Z), "overlap"), (dict(labels=W + 8), "overlap"),
    (dict(loss=A + 4), "overlap"), (dict(lse=B + N * K - 4), "overlap"), (dict(workspace=F), "overlap")])
def test_what_the_loss_refuses(wrong, word):
    assert xent(**wrong) == BAD and word in fp8.fp8_last_error(), fp8.fp8_last_error()


@pytest.mark.parametrize("wrong,word", [
    (dict(out_kind=4), "fp8_out_t"), (dict(D=None), "NULL"), (dict(out_kind=0, D=D + 2), "aligned"), (dict(out_kind=1, sD=F), "FP8 outputs"), (dict(amax=F + 2), "misaligned"),
    (dict(lse=None), "lse"), (dict(lse=Z + 1), "lse"), (dict(dloss=None), "dloss"), (dict(dloss=F + 2), "dloss"), (dict(ndloss=2), "ndloss"), (dict(ndloss=0), "ndloss"),
    (dict(D=A), "overlap"), (dict(D=B + N * K - 1), "overlap"), (dict(D=S), "overlap"), (dict(D=Z - 1), "overlap"), (dict(D=F + 64), "overlap")])
def test_what_the_gradient_refuses(wrong, word):
    assert grad(**wrong) == BAD and word in fp8.fp8_last_error(), fp8.fp8_last_error()


def test_sizes_beyond_what_bytes_can_be_counted():
    for call in (xent, grad):
        assert call(M=(1 << 40) + 1) == UNSUPPORTED
        assert call(M=1 << 35, N=1 << 35) == UNSUPPORTED


def test_more_rows_than_can_be_joined():
    """Refused before the product is launched, where a launch would fail for want of a device."""
    rows = 32 * ((1 << 32) // 256 - 1) + 1
    assert xent(M=rows, N=1, K=0, A=None, B=None, lse=Z + (1 << 36), workspace_bytes=1 << 40) == UNSUPPORTED and "grid limit" in fp8.fp8_last_error()


def test_workspace_size():
    size = fp8.fp8_gemm_xent_workspace_size
    assert [size(5, n) for n in (0, 1, 32, 33, 50257)] == [40, 80, 80, 120, 5 * 8 * (1571 + 1)]
    assert size(0, 10) == 0 and size(-1, 10) == 0 and size(10, -1) == 0
    for m, n in ((1 << 62, 1), (1 << 40, 1 << 40), ((1 << 63) - 1, (1 << 63) - 1)):
        assert size(m, n) == 2 ** 64 - 1
    assert size(1, (1 << 63) - 1) == 8 * ((1 << 58) + 1)


# ---- AdamW
def adamw(count=2, n=(200, 3), p=(A, A + 4096), p_dtype=(0, 1), g=(B, B + 4096), g_dtype=(1, 0), m=(D, D + 4096), v=(D + 8192, D + 12288), state_kind=0, m_scale=None, v_scale=None,
          weight_decay=None, lr=F, step=S, beta1=0.9, beta2=0.999, eps=1e-8, norm=None, max_norm=1.0, q=None, q_fmt=0, q_scale=None, q_amax=None, flags=0):
    def array(values, kind=vp):
        return values if values is None or isinstance(values, ctypes.Array) else (kind * max(1, len(values)))(*values)
    return L.fp8_adamw(count, array(p), array(p_dtype, ctypes.c_int), array(g), array(g_dtype, ctypes.c_int), array(n, ctypes.c_size_t), array(m), array(v), state_kind, array(m_scale),
                       array(v_scale), 1, array(weight_decay, ctypes.c_float), lr, step, beta1, beta2, eps, norm, max_norm, array(q), q_fmt, q_scale, q_amax, flags, None)


SCALES = dict(state_kind=1, m_scale=(Z, Z + 64), v_scale=(Z + 128, Z + 192))


@pytest.mark.parametrize("wrong,word", [
    (dict(count=-1), "negative"), (dict(p=None), "NULL"), (dict(g=None), "NULL"), (dict(n=None), "NULL"), (dict(m=None), "states"), (dict(v=None), "states"), (dict(p_dtype=(0, 2)), "fp8_dtype_t"),
    (dict(g_dtype=(-1, 0)), "fp8_dtype_t"), (dict(p=(A, None)), "NULL"), (dict(g=(None, B)), "NULL"), (dict(m=(D, None)), "m[1]"), (dict(v=(None, D)), "v[0]"), (dict(p=(A + 2, A + 4096)), "aligned"),
    (dict(p=(A, A + 4097)), "aligned"), (dict(g=(B, B + 4098)), "aligned"), (dict(m=(D + 2, D + 4096)), "misaligned"), (dict(state_kind=2), "fp8_state_t"), (dict(state_kind=1), "states"),
    (dict(SCALES, m_scale=(Z, None)), "m_scale[1]"), (dict(SCALES, v_scale=(Z + 2, Z + 64)), "v_scale[0]"), (dict(lr=None), "lr"), (dict(lr=F + 2), "lr"), (dict(step=None), "step"),
    (dict(step=S + 4), "step"), (dict(beta1=1.0), "beta"), (dict(beta1=-0.1), "beta"), (dict(beta2=1.0), "beta"), (dict(beta2=math.nan), "beta"), (dict(eps=-1e-8), "eps"), (dict(eps=math.inf), "eps"),
    (dict(weight_decay=(0.1, -0.1)), "weight_decay[1]"), (dict(weight_decay=(math.nan, 0.0)), "weight_decay[0]"), (dict(norm=F + 2), "norm"), (dict(norm=F, max_norm=-1.0), "max_norm"),
    (dict(norm=F, max_norm=math.nan), "max_norm"), (dict(q=(W, None)), "q_scale"), (dict(q=(W, None), q_scale=F, q_fmt=2), "fp8_format_t"), (dict(q=(W, None), q_scale=F + 1), "misaligned"),
    (dict(q_amax=F + 2), "misaligned"), (dict(flags=2), "flag"),
    # one tensor's own arguments in each other's memory, and one of the weights listed twice
    (dict(g=(A + 400, B)), "overlap"), (dict(m=(A, D)), "overlap"), (dict(v=(D, D + 12288)), "overlap"), (dict(q=(A + 799, None), q_scale=F), "overlap"),
    (dict(SCALES, v_scale=(Z + 4, Z + 192)), "overlap"), (dict(p=(A, A), p_dtype=(0, 0)), "two of the weights"), (dict(p=(A, A + 796), p_dtype=(0, 0)), "two of the weights")])
def test_what_adamw_refuses(wrong, word):
    assert adamw(**wrong) == BAD and word in fp8.fp8_last_error(), fp8.fp8_last_error()


def test_adamw_sizes():
    assert adamw(n=(200, (1 << 45) + 1)) == UNSUPPORTED and adamw(n=(200, (1 << 43) + 1)) == UNSUPPORTED
    # nothing to do: no pointer is looked at
    assert adamw(count=0, p=None, g=None, n=None, m=None, v=None, p_dtype=None, g_dtype=None) == fp8.FP8_OK
    assert adamw(n=(0, 0), p=(None, None), g=(None, None), m=(None, None), v=(None, None)) == fp8.FP8_OK
