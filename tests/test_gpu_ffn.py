"""The feed-forward operators on the GPU against a plain implementation in 64 bits: products with bias, activation and
residual, the gated block, both with their backward passes, in every kernel form.

Tolerances, from the operators' definition.  Products meet |c - c_ref| <= 2^-20 sum |a b| / (sA sB) (2^-10 with the FP8
instructions), E below.  No activation has a slope beyond 1.13.  With the exponential and the reciprocal of 1 ulp, a value
act(z) is off by at most 2^-19 |z|, a derivative by 2^-17 (1 - s, an ulp of 1 off, is multiplied by at most 20 before s is 1).
Each multiplication or addition behind that rounds once more (2^-23 of it); 2^-21 of the result covers them.  A stored value is
off by half an ulp more: 2^-8 of a bf16 one, 2^-4 / 2^-3 of an E4M3 / E5M2 one, or half the smallest subnormal."""
import contextlib
import math

import pytest
import torch

import paper_2209_05433_amd as fp8
from gpu_util import knob

pytestmark = pytest.mark.gpu

E4M3, E5M2 = fp8.FP8_E4M3, fp8.FP8_E5M2
TORCH8 = {E4M3: torch.float8_e4m3fn, E5M2: torch.float8_e5m2}
F32, BF16, O43, O52 = fp8.FP8_OUT_F32, fp8.FP8_OUT_BF16, fp8.FP8_OUT_E4M3, fp8.FP8_OUT_E5M2
ACTS = {"none": fp8.FP8_ACT_NONE, "relu": fp8.FP8_ACT_RELU, "gelu": fp8.FP8_ACT_GELU, "gelu_tanh": fp8.FP8_ACT_GELU_TANH, "silu": fp8.FP8_ACT_SILU}
WIDE = {F32: torch.float32, BF16: torch.bfloat16}

# what takes a call: the library's choice, plain FMAs, tiles of the small kernel, tiles of the tiled kernel
FORMS = {"chosen": {}, "fma": {fp8.FP8_KNOB_GEMM_KERNEL: 1}, "small_32x32": {fp8.FP8_KNOB_SMALL: 2}, "small_32x64": {fp8.FP8_KNOB_SMALL: 3},
         "small_64x64": {fp8.FP8_KNOB_SMALL: 4}, "tiled_256": {fp8.FP8_KNOB_SMALL: 1, fp8.FP8_KNOB_TILE_N: 256},
         "tiled_128": {fp8.FP8_KNOB_SMALL: 1, fp8.FP8_KNOB_TILE_N: 128}, "tiled_both": {fp8.FP8_KNOB_SMALL: 1, fp8.FP8_KNOB_MIXED: 2}}


@contextlib.contextmanager
def form(name):
    with contextlib.ExitStack() as stack:
        for k, v in FORMS[name].items():
            stack.enter_context(knob(k, v))
        yield


def value(z, act):
    if act == "none":
        return z
    if act == "relu":
        return torch.relu(z)
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))


def slope(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).double()
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (z + 0.044715 * z ** 3))
    return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)


class Guarded:
    """A buffer in the middle of a larger one whose other bytes must stay what they were."""
    PAD = 512

    def __init__(self, shape, dtype, shift=0):
        self.size = torch.tensor([], dtype=dtype).element_size()
        n = math.prod(shape) * self.size
        self.raw = torch.full((n + 2 * self.PAD + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        self.lo, self.hi = self.PAD + shift * self.size, self.PAD + shift * self.size + n
        self.t = self.raw[self.lo:self.hi].view(dtype).view(shape)

    def check(self):
        assert bool((self.raw[:self.lo] == 0xA5).all()) and bool((self.raw[self.hi:] == 0xA5).all()), "bytes beside the output were written"


def operand(gen, rows, cols, fmt, trans, shift=0):
    """(values [rows, cols] in 64 bits, bytes as stored)"""
    x = torch.randn(rows, cols, generator=gen, device="cuda") * (40.0 if fmt == E4M3 else 800.0)
    q = x.to(TORCH8[fmt])
    stored = (q.t() if trans else q).contiguous().view(torch.uint8)
    buf = torch.zeros(stored.numel() + 64, dtype=torch.uint8, device="cuda")
    buf[shift:shift + stored.numel()] = stored.flatten()
    return q.double(), buf[shift:shift + stored.numel()].view(stored.shape)


class Case:
    """Operands, factors and 64-bit sums of one product; wide: op(B) has 2 N columns."""

    def __init__(self, M, N, K, tA=False, tB=True, fA=E4M3, fB=E4M3, wide=False, per_row=False, factors="one", flags=0, shift=0, seed=0):
        gen = self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.M, self.N, self.K, self.tA, self.tB, self.fA, self.fB, self.flags, self.shift = M, N, K, tA, tB, fA, fB, flags, shift
        cols = 2 * N if wide else N
        a, self.A = operand(gen, M, K, fA, tA, shift)
        b, self.B = operand(gen, K, cols, fB, tB, shift)
        big = (40.0 if fA == E4M3 else 800.0) * (40.0 if fB == E4M3 else 800.0)
        scale = math.sqrt(big) * math.sqrt(math.sqrt(max(K, 1)))         # c comes out around 1
        draw = lambda n: scale * (0.5 + torch.rand(n, generator=gen, device="cuda"))
        self.sA = draw(M if per_row else 1)
        self.sB = draw({"one": 1, "pair": 2, "column": cols}[factors])
        fb = self.sB.double()
        if factors == "pair":
            fb = fb.repeat_interleave(N)
        per = self.sA.double().reshape(-1, 1) * fb.reshape(1, -1)
        self.c = (a @ b) / per if K else torch.zeros(M, cols, dtype=torch.float64, device="cuda") / per
        rel = 2.0 ** -10 if flags else 2.0 ** -20
        self.E = rel * ((a.abs() @ b.abs()) / per if K else torch.zeros_like(self.c)) + 2.0 ** -22 * self.c.abs()

    def randn(self, *shape, dtype=torch.float32):
        return torch.randn(shape, generator=self.gen, device="cuda").to(dtype)


def accept(got, kind, want, err, sD=1.0, what=""):
    """got: the stored output; want, err: 64-bit values and what they may be off before the rounding of the store."""
    if kind in WIDE:
        half = want.abs() * (2.0 ** -8 if kind == BF16 else 2.0 ** -24)
        bound = err + half + 1e-38
        g = got.double()
    else:
        fmt = E4M3 if kind == O43 else E5M2
        top, part, sub = (448.0, 2.0 ** -4, 2.0 ** -10) if fmt == E4M3 else (57344.0, 2.0 ** -3, 2.0 ** -17)
        v, e = want * sD, err * sD
        g = got.view(TORCH8[fmt]).double()
        want = v.clamp(-top, top)
        bound = e + torch.clamp((v.abs() + e) * part, min=sub)
    bad = ~((g - want).abs() <= bound)
    assert not bool(bad.any()), "%s: %d of %d off, worst at %s: %r for %r" % (
        what, int(bad.sum()), bad.numel(), tuple(bad.nonzero()[0].tolist()), float(g[bad][0]), float(want[bad][0]))


def out_tensor(shape, kind, shift=0):
    return Guarded(shape, WIDE.get(kind, torch.uint8), shift)


def check_amax(amax, want, err):
    assert abs(float(amax) - float(want.abs().max())) <= float(err.max()), "amax"


def factor_for(kind, want):
    if kind in WIDE:
        return None, 1.0
    s = torch.tensor([(448.0 if kind == O43 else 57344.0) / max(1e-6, 0.7 * float(want.abs().max()))], device="cuda")     # (the largest saturate)
    return s, float(s)


def run_act(c, act, kind, bias=None, residual=None, z=None, in_place=False, name="chosen", amax=True):
    M, N = c.M, c.N
    b = None if bias is None else c.randn(N, dtype=bias)
    r = None if residual is None else c.randn(M, N, dtype=residual)
    zw = c.c + (0 if b is None else b.double())
    want = value(zw, act) + (0 if r is None else r.double())
    err = 1.13 * c.E + 2.0 ** -19 * zw.abs() + 2.0 ** -21 * want.abs()
    sD, s = factor_for(kind, want) if want.numel() else (None, 1.0)
    D = out_tensor((M, N), kind, c.shift)
    if in_place:
        D.t.copy_(r)
    Z = None if z is None else Guarded((M, N), z, c.shift)
    top = torch.full((1,), -7.0, device="cuda") if amax else None
    with form(name):
        fp8.fp8_gemm_act(c.A, c.fA, c.tA, c.B, c.fB, c.tB, D.t, kind, c.sA, c.sB, ACTS[act], b, D.t if in_place else r, Z.t if Z else None, sD, top, c.flags)
    torch.cuda.synchronize()
    D.check()
    accept(D.t, kind, want, err, s, "D")
    if Z:
        Z.check()
        accept(Z.t, F32 if z == torch.float32 else BF16, zw, c.E + 2.0 ** -22 * zw.abs(), 1.0, "Z")
    if amax and want.numel():
        check_amax(top, want, err)
    return D.t


def run_act_grad(c, act, kind, z=torch.bfloat16, dbias=True, in_place=False, name="chosen"):
    M, N = c.M, c.N
    Z = (2 * c.randn(M, N)).to(z)
    Z.view(-1)[::7] = 0
    want = c.c * slope(Z.double(), act)
    err = 1.13 * c.E + 2.0 ** -17 * c.c.abs() + 2.0 ** -21 * want.abs()
    sD, s = factor_for(kind, want) if want.numel() else (None, 1.0)
    D = out_tensor((M, N), kind, c.shift)
    if in_place:
        D.t.copy_(Z)
    db = Guarded((N,), torch.float32) if dbias else None
    ws = Guarded((fp8.fp8_gemm_act_grad_workspace_size(M, N),), torch.uint8) if dbias else None
    top = torch.full((1,), -7.0, device="cuda")
    with form(name):
        fp8.fp8_gemm_act_grad(c.A, c.fA, c.tA, c.B, c.fB, c.tB, D.t, kind, c.sA, c.sB, ACTS[act], D.t if in_place else Z, db.t if db else None, ws.t if ws else None, sD, top, c.flags)
    torch.cuda.synchronize()
    D.check()
    accept(D.t, kind, want, err, s, "D")
    if want.numel():
        check_amax(top, want, err)
    if db:
        db.check()
        ws.check()
        # M additions in 32 bits: each at most 2^-24 of the sum so far
        accept(db.t, F32, want.sum(0), err.sum(0) + M * 2.0 ** -24 * want.abs().sum(0), 1.0, "dbias")
    return D.t, db.t if db else None


def run_gated(c, act, kind, gu=torch.bfloat16, name="chosen"):
    M, F = c.M, c.N
    g, u = c.c[:, :F], c.c[:, F:]
    want = value(g, act) * u
    eg, eu = c.E[:, :F], c.E[:, F:]
    ev = 1.13 * eg + 2.0 ** -19 * g.abs()
    err = ev * (u.abs() + eu) + value(g, act).abs() * eu + 2.0 ** -21 * want.abs()
    sD, s = factor_for(kind, want) if want.numel() else (None, 1.0)
    H = out_tensor((M, F), kind, c.shift)
    GU = None if gu is None else Guarded((M, 2 * F), gu, c.shift)
    top = torch.full((1,), -7.0, device="cuda")
    with form(name):
        fp8.fp8_gemm_gated(c.A, c.fA, c.tA, c.B, c.fB, c.tB, H.t, kind, c.sA, c.sB, ACTS[act], GU.t if GU else None, sD, top, c.flags)
    torch.cuda.synchronize()
    H.check()
    accept(H.t, kind, want, err, s, "H")
    if GU:
        GU.check()
        accept(GU.t, F32 if gu == torch.float32 else BF16, c.c, c.E, 1.0, "GU")
    if want.numel():
        check_amax(top, want, err)
    return H.t


def run_gated_grad(c, act, kind, gu=torch.bfloat16, in_place=False, name="chosen"):
    M, F = c.M, c.N
    GU = (2 * c.randn(M, 2 * F)).to(gu)
    g, u = GU.double()[:, :F], GU.double()[:, F:]
    want = torch.cat([c.c * u * slope(g, act), c.c * value(g, act)], 1)
    err = torch.cat([u.abs() * (1.13 * c.E + 2.0 ** -17 * c.c.abs()), value(g, act).abs() * c.E + 2.0 ** -19 * g.abs() * c.c.abs()], 1) + 2.0 ** -21 * want.abs()
    sD, s = factor_for(kind, want) if want.numel() else (None, 1.0)
    D = out_tensor((M, 2 * F), kind, c.shift)
    if in_place:
        D.t.copy_(GU)
    top = torch.full((1,), -7.0, device="cuda")
    with form(name):
        fp8.fp8_gemm_gated_grad(c.A, c.fA, c.tA, c.B, c.fB, c.tB, D.t, kind, c.sA, c.sB, ACTS[act], D.t if in_place else GU, sD, top, c.flags)
    torch.cuda.synchronize()
    D.check()
    accept(D.t, kind, want, err, s, "dGU")
    if want.numel():
        check_amax(top, want, err)
    return D.t


# Sizes: single rows and columns, edges inside and at a tile, K below, at and beyond the chunks and stages; orders of both operands
SIZES = [(1, 1, 1), (1, 64, 128), (3, 5, 7), (16, 48, 64), (33, 65, 100), (64, 128, 256), (100, 272, 384), (129, 320, 528), (257, 144, 1040), (300, 520, 1280)]
ORDERS = [(False, True), (False, False), (True, False), (True, True)]


@pytest.mark.parametrize("name", list(FORMS))
@pytest.mark.parametrize("M,N,K", SIZES)
def test_products_with_bias_activation_and_residual(M, N, K, name):
    for i, (tA, tB) in enumerate(ORDERS):
        for j, (kind, act) in enumerate([(BF16, "gelu"), (F32, "silu"), (O43, "relu"), (O52, "gelu_tanh"), (F32, "none")]):
            c = Case(M, N, K, tA, tB, fB=E5M2 if j == 3 else E4M3, per_row=j == 1, factors="column" if j in (1, 2) else "one", flags=(i + j) % 2, seed=7 * i + j)
            run_act(c, act, kind, bias=[torch.bfloat16, torch.float32, None][(i + j) % 3], residual=[None, torch.float32, torch.bfloat16][j % 3],
                    z=[torch.bfloat16, None, torch.float32][(i + 2 * j) % 3], name=name)


@pytest.mark.parametrize("name", list(FORMS))
@pytest.mark.parametrize("M,N,K", SIZES)
def test_gradient_through_activation_and_bias(M, N, K, name):
    for i, (tA, tB) in enumerate(ORDERS):
        for j, (kind, act) in enumerate([(O52, "gelu"), (F32, "silu"), (BF16, "relu"), (BF16, "gelu_tanh"), (O43, "none")]):
            c = Case(M, N, K, tA, tB, fA=E5M2, per_row=j == 1, factors="column" if j in (1, 2) else "one", flags=(i + j) % 2, seed=7 * i + j)
            run_act_grad(c, act, kind, z=[torch.bfloat16, torch.float32][(i + j) % 2], dbias=j != 3, name=name)


@pytest.mark.parametrize("name", list(FORMS))
@pytest.mark.parametrize("M,N,K", SIZES)
def test_gated_block(M, N, K, name):
    for i, (tA, tB) in enumerate(ORDERS):
        for j, (kind, act) in enumerate([(BF16, "silu"), (F32, "gelu"), (O43, "gelu_tanh"), (O52, "relu"), (F32, "none")]):
            c = Case(M, N, K, tA, tB, wide=True, per_row=j == 1, factors=["one", "column", "pair", "one", "pair"][j], flags=(i + j) % 2, seed=7 * i + j)
            run_gated(c, act, kind, gu=[torch.bfloat16, None, torch.float32][(i + j) % 3], name=name)


@pytest.mark.parametrize("name", list(FORMS))
@pytest.mark.parametrize("M,N,K", SIZES)
def test_gated_block_gradient(M, N, K, name):
    for i, (tA, tB) in enumerate(ORDERS):
        for j, (kind, act) in enumerate([(O52, "silu"), (F32, "gelu"), (BF16, "gelu_tanh"), (BF16, "relu"), (O43, "none")]):
            c = Case(M, N, K, tA, tB, fA=E5M2, per_row=j == 1, factors="column" if j in (1, 2) else "one", flags=(i + j) % 2, seed=7 * i + j)
            run_gated_grad(c, act, kind, gu=[torch.bfloat16, torch.float32][(i + j) % 2], name=name)


@pytest.mark.parametrize("M,N,K", [(700, 1000, 2048), (1537, 768, 640), (40, 2064, 4096), (2, 6144, 2048), (513, 4112, 272)])
def test_larger_products_by_the_librarys_choice(M, N, K):
    for flags in (0, fp8.FP8_GEMM_MFMA8):
        run_act(Case(M, N, K, flags=flags, seed=1), "gelu", O43, bias=torch.bfloat16, z=torch.bfloat16)
        run_act_grad(Case(M, N, K, tB=False, fA=E5M2, flags=flags, seed=2), "gelu", O52)
        run_gated(Case(M, N, K, wide=True, flags=flags, seed=3), "silu", BF16)
        run_gated_grad(Case(M, N, K, tB=False, fA=E5M2, flags=flags, seed=4), "silu", O52)


@pytest.mark.parametrize("name", ["chosen", "tiled_256", "tiled_128", "tiled_both"])
@pytest.mark.parametrize("M,N,K", [(272, 144, 100), (528, 272, 333), (256, 512, 33), (16, 32, 129)])
def test_any_k_where_no_operand_is_contiguous_along_it(M, N, K, name):
    for flags in (0, fp8.FP8_GEMM_MFMA8):
        order = dict(tA=True, tB=False, flags=flags)
        run_act(Case(M, N, K, seed=21, **order), "gelu", BF16, bias=torch.float32, residual=torch.bfloat16, name=name)
        run_act_grad(Case(M, N, K, fA=E5M2, seed=22, **order), "silu", O52, name=name)
        run_gated(Case(M, N, K, wide=True, seed=23, **order), "silu", O43, name=name)
        run_gated_grad(Case(M, N, K, fA=E5M2, seed=24, **order), "gelu", F32, gu=torch.float32, name=name)


@pytest.mark.parametrize("name", list(FORMS))
def test_in_place(name):
    """The residual, z or g | u where the output goes."""
    for kind, dtype in ((BF16, torch.bfloat16), (F32, torch.float32)):
        run_act(Case(130, 200, 96, seed=5), "gelu", kind, residual=dtype, in_place=True, name=name)
        run_act_grad(Case(130, 200, 96, seed=6), "silu", kind, z=dtype, in_place=True, name=name)
        run_gated_grad(Case(130, 200, 96, seed=7), "silu", kind, gu=dtype, in_place=True, name=name)


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_tensors_that_start_anywhere(shift):
    """Operands at any byte, outputs and tensors beside them at any element."""
    for M, N, K in ((37, 90, 160), (260, 144, 256)):
        run_act(Case(M, N, K, shift=shift, seed=8), "gelu", BF16, bias=torch.bfloat16, residual=torch.bfloat16, z=torch.bfloat16)
        run_act(Case(M, N, K, shift=shift, seed=8), "gelu", O43, z=torch.float32)
        run_act_grad(Case(M, N, K, tB=False, shift=shift, seed=9), "gelu", F32)
        run_gated(Case(M, N, K, wide=True, shift=shift, seed=10), "silu", O43)
        run_gated(Case(M, N, K, tB=False, wide=True, shift=shift, seed=10), "silu", BF16)
        run_gated_grad(Case(M, N, K, tB=False, shift=shift, seed=11), "silu", BF16)


@pytest.mark.parametrize("name", ["chosen", "small_64x64", "fma"])
def test_tensors_beyond_32_bits_of_elements(name):
    """Outputs and the tensors beside them of 2.3e9 elements; the first and the last 300 rows hold something (the other sums are 0)."""
    M, R, N, K = 140001, 300, 16400, 32
    F = N // 2
    ends = (slice(0, R), slice(M - R, M))

    def operands(wide, n, fA, seed):
        c = Case(R, n, K, fA=fA, wide=wide, seed=seed)
        A = torch.zeros(M, K, dtype=torch.uint8, device="cuda")
        for e in ends:
            A[e] = c.A
        return c, A

    def beside(c, cols):
        x = (2 * c.randn(R, cols)).bfloat16()
        t = torch.zeros(M, cols, dtype=torch.bfloat16, device="cuda")
        for e in ends:
            t[e] = x
        return x.double(), t

    D = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    Z = torch.empty_like(D)
    with form(name):
        c, A = operands(False, N, E4M3, 31)
        r, res = beside(c, N)
        fp8.fp8_gemm_act(A, E4M3, False, c.B, E4M3, True, D, BF16, c.sA, c.sB, ACTS["gelu"], None, res, Z)
        want = value(c.c, "gelu") + r
        for e in ends:
            accept(D[e], BF16, want, 1.13 * c.E + 2.0 ** -19 * c.c.abs() + 2.0 ** -21 * want.abs(), what="D")
            accept(Z[e], BF16, c.c, c.E, what="Z")
        assert not bool(D[M // 2 - 500:M // 2 + 500].any())

        c, A = operands(False, N, E5M2, 32)
        z, side = beside(c, N)
        db = torch.empty(N, device="cuda")
        ws = torch.empty(fp8.fp8_gemm_act_grad_workspace_size(M, N), dtype=torch.uint8, device="cuda")
        fp8.fp8_gemm_act_grad(A, E5M2, False, c.B, E4M3, True, D, BF16, c.sA, c.sB, ACTS["gelu"], side, db, ws)
        want = c.c * slope(z, "gelu")
        err = 1.13 * c.E + 2.0 ** -17 * c.c.abs() + 2.0 ** -21 * want.abs()
        for e in ends:
            accept(D[e], BF16, want, err, what="dZ")
        accept(db, F32, 2 * want.sum(0), 2 * (err.sum(0) + M * 2.0 ** -24 * want.abs().sum(0)), what="dbias")
        assert not bool(D[M // 2 - 500:M // 2 + 500].any())
        del side, res

        c, A = operands(True, F, E4M3, 33)
        H = torch.empty(M, F, dtype=torch.bfloat16, device="cuda")
        fp8.fp8_gemm_gated(A, E4M3, False, c.B, E4M3, True, H, BF16, c.sA, c.sB, ACTS["silu"], Z)
        g, u = c.c[:, :F], c.c[:, F:]
        want = value(g, "silu") * u
        eg, eu = c.E[:, :F], c.E[:, F:]
        err = (1.13 * eg + 2.0 ** -19 * g.abs()) * (u.abs() + eu) + value(g, "silu").abs() * eu + 2.0 ** -21 * want.abs()
        for e in ends:
            accept(H[e], BF16, want, err, what="H")
            accept(Z[e], BF16, c.c, c.E, what="GU")
        del H

        c, A = operands(False, F, E5M2, 34)
        gu, side = beside(c, N)
        fp8.fp8_gemm_gated_grad(A, E5M2, False, c.B, E4M3, True, D, BF16, c.sA, c.sB, ACTS["silu"], side)
        g, u = gu[:, :F], gu[:, F:]
        want = torch.cat([c.c * u * slope(g, "silu"), c.c * value(g, "silu")], 1)
        err = torch.cat([u.abs() * (1.13 * c.E + 2.0 ** -17 * c.c.abs()), value(g, "silu").abs() * c.E + 2.0 ** -19 * g.abs() * c.c.abs()], 1) + 2.0 ** -21 * want.abs()
        for e in ends:
            accept(D[e], BF16, want, err, what="dGU")
        assert not bool(D[M // 2 - 500:M // 2 + 500].any())


def test_empty_products():
    run_act(Case(5, 0, 16), "gelu", BF16, bias=torch.bfloat16)
    run_act(Case(0, 24, 16), "gelu", BF16, bias=torch.bfloat16)
    run_act_grad(Case(0, 24, 16), "gelu", BF16)                       # dbias of no rows: zeros
    run_gated(Case(0, 8, 16, wide=True), "silu", BF16)
    run_gated_grad(Case(4, 0, 16), "silu", BF16)
    # no products at all: the sums are 0, everything behind them still happens
    run_act(Case(70, 33, 0), "gelu", BF16, bias=torch.float32, residual=torch.float32, z=torch.float32)
    run_act_grad(Case(70, 33, 0), "gelu", F32)
    run_gated(Case(70, 33, 0, wide=True), "silu", O43)
    run_gated_grad(Case(70, 33, 0), "silu", BF16)


GRID = [0.0, -0.0, 1e-30, -1e-30, 1e-4, -1e-4, 0.5, -0.5, 1.0, -1.0, 1.7, -1.7, 3.0, -3.0, 5.5, -5.5, 9.0, -9.0, 15.9, -15.9, 16.1, -16.1, 50.0, -50.0,
        120.0, -120.0, 130.0, -130.0, 1e10, -1e10, 3e38, -3e38]


@pytest.mark.parametrize("act", list(ACTS))
def test_activations_and_their_derivatives_over_the_whole_range(act):
    """A product of ones makes the operators the activation itself: against the formula, and its derivative against differences."""
    z = torch.cat([torch.tensor(GRID, device="cuda"), torch.linspace(-20, 20, 4001, device="cuda")]).reshape(1, -1)
    N = z.numel()
    one = torch.full((1, 1), 0x38, dtype=torch.uint8, device="cuda")                    # 1.0 in E4M3
    ones, s1 = one.expand(1, N).contiguous(), torch.ones(1, device="cuda")
    got, zero = torch.empty(1, N, device="cuda"), torch.zeros(1, 1, dtype=torch.uint8, device="cuda")
    # act(z): the product is 0, the bias z
    fp8.fp8_gemm_act(zero, E4M3, False, ones, E4M3, False, got, F32, s1, s1, ACTS[act], z.reshape(-1))
    zd = z.double()
    assert bool(((got.double() - value(zd, act)).abs() <= 2.0 ** -19 * zd.abs()).all())
    # act'(z): the gradient is 1
    fp8.fp8_gemm_act_grad(one, E4M3, False, ones, E4M3, False, got, F32, s1, s1, ACTS[act], z)
    h = 1e-5
    fine = zd.abs() > 2 * h if act == "relu" else torch.ones_like(zd, dtype=torch.bool)
    near = zd.abs() <= 1e4                                                                # (a step of h is not lost in z)
    exact = slope(zd.clamp(-1e4, 1e4), act)
    assert bool(((got.double() - exact).abs() <= 2.0 ** -17).all())
    difference = (value(zd + h, act) - value(zd - h, act)) / (2 * h)
    # (truncation h^2 / 6 times the third derivative, below 1, and rounding 2^-53 |z| / h)
    assert bool(((got.double() - difference).abs() <= 2.0 ** -17 + h * h + 2.0 ** -50 * zd.abs() / h)[fine & near].all())


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
def test_gated_gradient_against_differences(act):
    """d/dg and d/du of act(g) u, by differences of the formula in 64 bits; the incoming gradient is 1."""
    g = torch.linspace(-8, 8, 101, device="cuda").repeat_interleave(9)
    u = torch.linspace(-3, 3, 9, device="cuda").repeat(101)
    F = g.numel()
    GU = torch.cat([g, u]).reshape(1, -1).contiguous()
    one = torch.full((1, 1), 0x38, dtype=torch.uint8, device="cuda")
    s1, got = torch.ones(1, device="cuda"), torch.empty(1, 2 * F, device="cuda")
    fp8.fp8_gemm_gated_grad(one, E4M3, False, one.expand(1, F).contiguous(), E4M3, False, got, F32, s1, s1, ACTS[act], GU)
    gd, ud, h = g.double(), u.double(), 1e-5
    dg = (value(gd + h, act) - value(gd - h, act)) / (2 * h) * ud
    du = value(gd, act)
    fine = gd.abs() > 2 * h
    assert bool(((got[0, :F].double() - dg).abs() <= 3 * (2.0 ** -17 + 1e-8) )[fine].all())
    assert bool(((got[0, F:].double() - du).abs() <= 2.0 ** -19 * gd.abs() + 2.0 ** -21 * du.abs()).all())


@pytest.mark.parametrize("name", list(FORMS))
def test_nan_and_infinity(name):
    """A NaN in an operand reaches the outputs of its row and no others, the maximum is NaN; an infinite pre-activation gives the limits."""
    M, N, K = 70, 96, 128
    c = Case(M, N, K, fA=E5M2, seed=3)
    c.A[17, 5] = 0x7F
    D, top = torch.empty(M, N, device="cuda"), torch.zeros(1, device="cuda")
    with form(name):
        fp8.fp8_gemm_act(c.A, E5M2, False, c.B, E4M3, True, D, F32, c.sA, c.sB, ACTS["relu"], None, None, None, None, top)
        assert bool(D[17].isnan().all()) and not bool(D[:17].isnan().any()) and not bool(D[18:].isnan().any()) and bool(top.isnan().all())
        H = torch.empty(M, N // 2, device="cuda", dtype=torch.uint8)
        fp8.fp8_gemm_gated(c.A, E5M2, False, c.B, E4M3, True, H, O43, c.sA, c.sB, ACTS["silu"], None, None, top)
        assert bool((H[17] & 0x7F == 0x7F).all()) and not bool((H[18:] & 0x7F == 0x7F).any()) and bool(top.isnan().all())
        inf = torch.full((N,), float("inf"), device="cuda")
        for act in ("relu", "gelu", "gelu_tanh", "silu"):
            c2 = Case(M, N, K, seed=4)
            for bias, limit in ((inf, float("inf")), (-inf, 0.0)):
                fp8.fp8_gemm_act(c2.A, E4M3, False, c2.B, E4M3, True, D, F32, c2.sA, c2.sB, ACTS[act], bias)
                assert bool((D == limit).all()), (act, limit)
            for z, limit in ((inf, 1.0), (-inf, 0.0)):
                fp8.fp8_gemm_act_grad(c2.A, E4M3, False, c2.B, E4M3, True, D, F32, c2.sA, c2.sB, ACTS[act], z.expand(M, N).contiguous())
                assert bool(((D.double() - limit * c2.c).abs() <= c2.E + 2.0 ** -24 * c2.c.abs()).all()), (act, limit)
            fp8.fp8_gemm_act_grad(c2.A, E4M3, False, c2.B, E4M3, True, D, F32, c2.sA, c2.sB, ACTS[act], torch.full((M, N), float("nan"), device="cuda"))
            assert bool(D.isnan().all()), act


@pytest.mark.parametrize("name", list(FORMS))
@pytest.mark.parametrize("M", [3, 70])
def test_an_infinity_at_the_end_of_k_gives_infinite_sums(M, name):
    """K = 272 fills no chunk, trip or stage: what stands in for the rest has to leave the sums alone."""
    N, K = 48, 272
    for tB in (True, False):
        c = Case(M, N, K, tB=tB, fA=E5M2, fB=E5M2, seed=12)
        c.A[:, K - 1] = 0x3C                                    # 1.0 against the infinity
        (c.B[5] if tB else c.B[:, 5])[K - 1] = 0x7C
        want = torch.zeros(M, N, dtype=torch.bool, device="cuda")
        want[:, 5] = True
        D = torch.empty(M, N, device="cuda")
        G = torch.empty(M, N // 2, device="cuda")
        GU = torch.empty(M, N, device="cuda")
        with form(name):
            fp8.fp8_gemm_act(c.A, E5M2, False, c.B, E5M2, tB, D, F32, c.sA, c.sB, ACTS["none"])
            fp8.fp8_gemm_gated(c.A, E5M2, False, c.B, E5M2, tB, G, F32, c.sA, c.sB, ACTS["none"], GU)
        assert torch.equal(D == float("inf"), want) and torch.equal(D.isfinite(), ~want)
        assert torch.equal(GU == float("inf"), want) and torch.equal(GU.isfinite(), ~want)


@pytest.mark.parametrize("name", list(FORMS))
def test_sums_are_the_same_in_every_run(name):
    c = Case(500, 272, 512, tB=False, seed=9)
    runs = []
    for _ in range(3):
        c.gen.manual_seed(77)
        runs.append([t.clone() for t in run_act_grad(c, "gelu", F32, name=name)])
    for r in runs[1:]:
        assert torch.equal(r[0], runs[0][0]) and torch.equal(r[1], runs[0][1])


@pytest.mark.parametrize("M,N,K", [(1, 2048, 6144), (1, 1000, 1008), (5, 77, 4112), (16, 4096, 2048), (13, 2000, 272), (16, 16, 16), (2, 17, 8192)])
def test_a_few_rows(M, N, K):
    for flags in (0, fp8.FP8_GEMM_MFMA8):
        for fB in (E4M3, E5M2):
            run_act(Case(M, N, K, fB=fB, flags=flags, per_row=True, factors="column", seed=1), "gelu", BF16, bias=torch.bfloat16, residual=torch.float32, z=torch.float32)
            run_act(Case(M, N, K, fB=fB, flags=flags, seed=2), "silu", O43)
            run_act_grad(Case(M, N, K, fA=E5M2, fB=fB, flags=flags, seed=3), "gelu_tanh", O52)
            run_gated(Case(M, N // 2, K, wide=True, fB=fB, factors="pair", flags=flags, seed=4), "silu", O43)
            run_gated_grad(Case(M, N, K, fA=E5M2, fB=fB, flags=flags, seed=5), "silu", F32, gu=torch.float32)


def test_another_stream_and_graph_replays():
    c = Case(300, 256, 512, wide=True, seed=12)
    GU, H = torch.empty(300, 512, device="cuda"), torch.empty(300, 256, device="cuda")
    call = lambda: fp8.fp8_gemm_gated(c.A, E4M3, False, c.B, E4M3, True, H, F32, c.sA, c.sB, ACTS["silu"], GU, None, None)
    call()
    torch.cuda.synchronize()
    want = H.clone(), GU.clone()
    stream = torch.cuda.Stream()
    H.zero_(); GU.zero_()
    torch.cuda.synchronize()
    fp8.fp8_gemm_gated(c.A, E4M3, False, c.B, E4M3, True, H, F32, c.sA, c.sB, ACTS["silu"], GU, None, None, 0, stream)
    stream.synchronize()
    assert torch.equal(H, want[0]) and torch.equal(GU, want[1])
    Z, D = c.randn(300, 512), torch.empty(300, 512, device="cuda")
    db, ws, top = torch.empty(512, device="cuda"), torch.empty(fp8.fp8_gemm_act_grad_workspace_size(300, 512), dtype=torch.uint8, device="cuda"), torch.empty(1, device="cuda")
    both = lambda: (call(), fp8.fp8_gemm_act_grad(c.A, E4M3, False, c.B, E4M3, True, D, F32, c.sA, c.sB, ACTS["gelu"], Z, db, ws, None, top))
    both()
    torch.cuda.synchronize()
    eager = [t.clone() for t in (H, GU, D, db, top)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for t in (H, GU, D, db, top):
            t.fill_(-3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((H, GU, D, db, top), eager))


def test_outputs_that_are_lazy_clones_leave_their_origin_alone():
    """As for the other entry points (tests/test_gpu_binding.py): every tensor that a call writes gets memory of its own first."""
    c, wide = Case(64, 32, 96, seed=20), Case(64, 32, 96, wide=True, seed=21)
    f32 = lambda *s: torch.full(s, 7.0, device="cuda")
    u8 = lambda *s: torch.full(s, 7, dtype=torch.uint8, device="cuda")
    Z, GU, norm, act = torch.randn(64, 32, device="cuda"), torch.randn(64, 64, device="cuda"), torch.full((1,), 3.0, device="cuda"), ACTS["silu"]
    need = fp8.fp8_gemm_act_grad_workspace_size(64, 32)
    zeros = lambda: torch.zeros(fp8.FP8_GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    calls = {
        "fp8_gemm_act": ([u8(64, 32), f32(64, 32), f32(1)],
                         lambda o: fp8.fp8_gemm_act(c.A, E4M3, False, c.B, E4M3, True, o[0], O43, c.sA, c.sB, act, None, None, o[1], None, o[2])),
        "fp8_gemm_act_grad": ([f32(64, 32), f32(32), u8(need), f32(1)],
                              lambda o: fp8.fp8_gemm_act_grad(c.A, E4M3, False, c.B, E4M3, True, o[0], F32, c.sA, c.sB, act, Z, o[1], o[2], None, o[3])),
        "fp8_gemm_gated": ([f32(64, 32), f32(64, 64), f32(1)],
                           lambda o: fp8.fp8_gemm_gated(wide.A, E4M3, False, wide.B, E4M3, True, o[0], F32, wide.sA, wide.sB, act, o[1], None, o[2])),
        "fp8_gemm_gated_grad": ([f32(64, 64), f32(1)],
                                lambda o: fp8.fp8_gemm_gated_grad(c.A, E4M3, False, c.B, E4M3, True, o[0], F32, c.sA, c.sB, act, GU, None, o[1])),
        "fp8_grad_norm": ([f32(1), zeros()], lambda o: fp8.fp8_grad_norm([Z, GU], o[0], o[1])),
        "fp8_grad_clip": ([f32(64, 32), f32(64, 64)], lambda o: fp8.fp8_grad_clip([Z, GU], norm, 1.0, o)),
    }
    assert set(calls) == set(fp8.binding.OPERATOR_CALLS)
    for name, (origins, call) in calls.items():
        before, clones, plain = [t.clone() for t in origins], [torch._lazy_clone(t) for t in origins], [t.clone() for t in origins]
        call(clones)
        call(plain)
        torch.cuda.synchronize()
        assert all(torch.equal(t, b) for t, b in zip(origins, before)), name
        assert all(torch.equal(a, b) for a, b in zip(clones, plain)), name
    x = f32(100)
    lazy = torch._lazy_clone(x)                              # in place: the clone changes, its origin does not
    fp8.fp8_grad_clip([lazy], norm, 1.0)
    torch.cuda.synchronize()
    assert bool((x == 7.0).all()) and bool((lazy < 7.0).all())


def test_arguments_that_do_not_fit():
    c, D = Case(8, 16, 32, seed=22), torch.empty(8, 16, device="cuda")
    good = lambda **k: fp8.fp8_gemm_act(**{**dict(A=c.A, fmtA=E4M3, transA=False, B=c.B, fmtB=E4M3, transB=True, D=D, out_kind=F32, sA=c.sA, sB=c.sB, act=0), **k})
    good()
    for k in (dict(A=c.A.float()), dict(B=c.B[:, :16]), dict(D=D[:, :8]), dict(D=D.half()), dict(out_kind=BF16), dict(sA=c.sA.double()), dict(bias=torch.zeros(15, device="cuda")),
              dict(bias=torch.zeros(16)), dict(residual=D.t()), dict(Z=torch.zeros(8, 15, device="cuda")), dict(sD=torch.ones(2, device="cuda"), out_kind=F32), dict(D=torch.empty(8, 32, device="cuda")[:, ::2])):
        with pytest.raises(ValueError):
            good(**k)
    with pytest.raises(TypeError):
        good(bias=torch.zeros(16, dtype=torch.float16, device="cuda"))
    with pytest.raises(TypeError):
        good(act="gelu")
    for k in (dict(act=7), dict(flags=8), dict(fmtA=3), dict(sD=torch.ones(1, device="cuda"))):
        with pytest.raises(fp8.Fp8Error) as e:
            good(**k)
        assert e.value.status == fp8.FP8_ERR_INVALID_ARG
    with pytest.raises(ValueError):                          # an odd number of columns for pairs
        fp8.fp8_gemm_gated(c.A, E4M3, False, c.B[:15].contiguous(), E4M3, True, torch.empty(8, 7, device="cuda"), F32, c.sA, c.sB, 4)
    with pytest.raises(TypeError):
        fp8.fp8_gemm_gated_grad(c.A, E4M3, False, c.B, E4M3, True, torch.empty(8, 32, device="cuda"), F32, c.sA, c.sB, 4, None)
    with pytest.raises(ValueError):
        fp8.fp8_grad_norm([D], torch.zeros(1, device="cuda"), torch.zeros(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(TypeError):
        fp8.fp8_grad_norm([D.half()], torch.zeros(1, device="cuda"), torch.zeros(1 << 15, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        fp8.fp8_grad_clip([D], torch.ones(1, device="cuda"), 1.0, [D.bfloat16()])


# ---- norm and clipping of gradients ------------------------------------------------------------------------------------------
def gradients(sizes, seed, offset=0):
    """Tensors of the given sizes, 16 and 32 bits in turn, each starting at an element of its own choice."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        dtype = torch.bfloat16 if i % 2 else torch.float32
        t = torch.randn(n + 8, generator=gen, device="cuda").mul_(0.01).to(dtype)
        out.append(t[(offset * i) % 8:][:n])
    return out


CLIP_SIZES = [[], [0], [1], [0, 0, 5, 0], [7, 8, 9], [16384], [16383, 16385, 0, 1], [100000, 3, 250007], [1 + 37 * i for i in range(700)], [(1 << 22) + 5, 12, 1 << 20]]


@pytest.mark.parametrize("sizes", CLIP_SIZES, ids=lambda s: "%d_tensors_%d" % (len(s), sum(s)))
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_gradient_norm_and_clipping(sizes, offset):
    xs = gradients(sizes, 5, offset)
    ws = torch.zeros(fp8.FP8_GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    norm = torch.full((1,), -1.0, device="cuda")
    want = math.sqrt(sum(float(x.double().square().sum()) for x in xs))
    for _ in range(2):                                       # (the workspace is ready for the next call)
        fp8.fp8_grad_norm(xs, norm, ws)
        assert abs(float(norm) - want) <= 2.0 ** -23 * want
    first = norm.clone()
    fp8.fp8_grad_norm(xs, norm, ws)
    assert torch.equal(first, norm)
    for most in (0.5 * want, 2 * want + 1, 0.0):
        f = torch.tensor(most, dtype=torch.float32, device="cuda") / (norm + 1e-6)
        f = f.clamp(max=1.0)
        outs = [Guarded((x.numel(),), x.dtype, offset % 4) for x in xs]
        fp8.fp8_grad_clip(xs, norm, most, [o.t for o in outs])
        # (the factor: a division that is right to an ulp; products are rounded once)
        for x, o in zip(xs, outs):
            o.check()
            ref = x.double() * f.double()
            half = 2.0 ** -8 if x.dtype == torch.bfloat16 else 2.0 ** -24
            assert bool(((o.t.double() - ref).abs() <= ref.abs() * (half + 2.0 ** -22) + 1e-40).all())
        mine = [x.clone() for x in xs]
        fp8.fp8_grad_clip(mine, norm, most)
        assert all(torch.equal(m, o.t) for m, o in zip(mine, outs))


def test_gradient_norm_of_large_small_and_special_values():
    ws = torch.zeros(fp8.FP8_GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    norm = torch.empty(1, device="cuda")
    x = torch.full((70000,), 3e30, device="cuda")            # squares beyond 32 bits
    y = torch.full((70000,), 1e-30, dtype=torch.bfloat16, device="cuda")
    fp8.fp8_grad_norm([x, y], norm, ws)
    assert abs(float(norm) / (3e30 * math.sqrt(70000)) - 1) < 2.0 ** -22
    fp8.fp8_grad_norm([y], norm, ws)
    assert abs(float(norm) / (float(y[0]) * math.sqrt(70000)) - 1) < 2.0 ** -22
    x[69999] = float("inf")
    z = x.clone()
    fp8.fp8_grad_norm([x, y], norm, ws)
    assert float(norm) == float("inf")
    fp8.fp8_grad_clip([z], norm, 1.0)
    assert bool((z[:-1] == 0).all()) and bool(z[-1].isnan())
    x[3] = float("nan")
    fp8.fp8_grad_norm([x, y], norm, ws)
    assert bool(norm.isnan())
    fp8.fp8_grad_clip([y], norm, 1.0)
    assert bool(y.isnan().all())
    fp8.fp8_grad_norm([torch.ones(5, device="cuda")], norm, ws)
    assert abs(float(norm) - math.sqrt(5)) < 1e-6


def test_clipping_beyond_32_bits_of_elements():
    n = (1 << 31) + 100003
    x = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(fp8.FP8_GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    norm = torch.empty(1, device="cuda")
    fp8.fp8_grad_norm([x], norm, ws)
    assert abs(float(norm) / (0.5 * math.sqrt(n)) - 1) < 2.0 ** -22
    fp8.fp8_grad_clip([x], norm, 0.5 * float(norm))
    assert float(x.min()) == 0.25 and float(x.max()) == 0.25


def test_clipping_in_a_graph():
    xs = gradients([3000, 70000, 17], 6)
    ws = torch.zeros(fp8.FP8_GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    norm, outs = torch.empty(1, device="cuda"), [torch.empty_like(x) for x in xs]
    step = lambda: (fp8.fp8_grad_norm(xs, norm, ws), fp8.fp8_grad_clip(xs, norm, 0.1, outs))
    step()
    torch.cuda.synchronize()
    eager = [norm.clone()] + [o.clone() for o in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        norm.fill_(0)
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, eager[0]) and all(torch.equal(o, e) for o, e in zip(outs, eager[1:]))
