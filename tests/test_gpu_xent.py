"""Cross entropy over a vocabulary behind its product, and its gradient, on the GPU against a plain implementation in 64 bits, in every kernel form.

Tolerances, with u = 2^-24, half a step of fp32.  A logit is off by E = 2^-20 sum |a b| / (sA sB) (2^-10 with the FP8 instructions) as that of any product.
The loss: t = z log2(e) is the sum times a rounded factor, 2u |z|; t - ref rounds once, u (|t| + |ref|), both at most max |z|: 2^-22 max |z| with the factor's; an exponential of
1 ulp is 2u, and a run of 16 terms and the two joins of four runs, lanes and halves at most 22 roundings of the sum, together 2^-19; lse itself rounds to u |lse|,
covered by 2^-22 |lse|.  loss: another E and 2u |z| for the label's logit, roundings of the difference, and 2 w |lse| times lse's error for the square.
The gradient: z log2(e) - lse log2(e) has the factors' roundings, 2u |z| + 2u |lse| + u |z - lse|, at most 2^-22 (|z| + |lse|); exponential, scale and product 8u; the
label's difference 2u dloss.  A stored value is off by half an ulp more: 2^-8 of a bf16 one, 2^-4 / 2^-3 of an E4M3 / E5M2 one, or half the smallest subnormal."""
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
DTYPE = {F32: torch.float32, BF16: torch.bfloat16, O43: torch.uint8, O52: torch.uint8}
FORMS = {"chosen": {}, "any_256": {fp8.FP8_KNOB_GEMM_KERNEL: 2, fp8.FP8_KNOB_TILE_N: 256},
         "any_128": {fp8.FP8_KNOB_GEMM_KERNEL: 2, fp8.FP8_KNOB_TILE_N: 128}, "fma": {fp8.FP8_KNOB_GEMM_KERNEL: 1}, "small_32x32": {fp8.FP8_KNOB_SMALL: 2}, "small_32x64": {fp8.FP8_KNOB_SMALL: 3},
         "small_64x64": {fp8.FP8_KNOB_SMALL: 4}, "tiled_256": {fp8.FP8_KNOB_SMALL: 1, fp8.FP8_KNOB_TILE_N: 256},
         "tiled_128": {fp8.FP8_KNOB_SMALL: 1, fp8.FP8_KNOB_TILE_N: 128}, "tiled_both": {fp8.FP8_KNOB_SMALL: 1, fp8.FP8_KNOB_MIXED: 2}}


@contextlib.contextmanager
def form(name):
    with contextlib.ExitStack() as stack:
        for k, v in FORMS[name].items():
            stack.enter_context(knob(k, v))
        yield


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


class Problem:
    def __init__(self, M, N, K, fa=E4M3, fb=E4M3, tA=False, tB=True, rows=False, columns=False, first=0, spread=2.5, seed=0, shift=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.M, self.N, self.K, self.fa, self.fb, self.tA, self.tB, self.first = M, N, K, fa, fb, tA, tB, first
        a = torch.randn((M, K), generator=g, device="cuda")
        b = torch.randn((N, K), generator=g, device="cuda") * (spread / math.sqrt(max(K, 1)))
        self.sA = 0.5 + 8 * torch.rand(M if rows else 1, generator=g, device="cuda")
        self.sB = 16 + 16 * torch.rand(N if columns else 1, generator=g, device="cuda")
        a8 = (a * self.sA[:, None]).clamp(-448, 448).to(TORCH8[fa])
        b8 = (b * self.sB[:, None]).clamp(-448, 448).to(TORCH8[fb])
        self.set(a8, b8, shift)
        self.labels = torch.randint(0, 2 * first + N if N else 5, (M,), generator=g, device="cuda")
        if M > 3:
            self.labels[torch.rand(M, generator=g, device="cuda") < 0.2] = -100
            self.labels[1] = first + N - 1                      # the last column, the first, one behind the piece
            self.labels[2] = first
            self.labels[3] = first + N

    def set(self, a8, b8, shift=0):
        def stored(x, trans):
            x = (x.t() if trans else x).contiguous().view(torch.uint8)
            buffer = torch.empty(x.numel() + shift, dtype=torch.uint8, device="cuda")
            buffer[shift:] = x.reshape(-1)
            return buffer[shift:].view(x.shape)
        self.A, self.B = stored(a8, self.tA), stored(b8, not self.tB)
        a, b = a8.double(), b8.double()
        scale = self.sA.double()[:, None] * self.sB.double()[None, :]
        self.z = (a @ b.t().contiguous()) / scale
        self.sizes = (a.abs() @ b.abs().t().contiguous()) / scale

    @property
    def bound(self):
        return 2.0 ** -20 * self.sizes

    def loss(self, z_weight=0.0, flags=0, stream=None, into=None):
        loss, lse = into or (Guarded((self.M,), torch.float32), Guarded((self.M,), torch.float32))
        ws = Guarded((fp8.fp8_gemm_xent_workspace_size(self.M, self.N) // 8,), torch.int64)
        fp8.fp8_gemm_xent(self.A, self.fa, self.tA, self.B, self.fb, self.tB, self.labels, loss.t, lse.t, ws.t, self.sA, self.sB, self.first, z_weight, flags, stream)
        for x in (loss, lse, ws):
            x.check()
        return loss.t, lse.t

    def expected_loss(self, z_weight=0.0, bits=20):
        """(loss, its tolerance, lse, its tolerance)"""
        z, E = self.z, 2.0 ** -bits * self.sizes
        lse = torch.logsumexp(z, 1)
        top = z.abs().amax(1)
        tol = E.amax(1) + 2.0 ** -22 * (lse.abs() + top) + 2.0 ** -19
        column = self.labels - self.first
        here = (column >= 0) & (column < self.N)
        at = torch.where(here, column, 0)[:, None]
        target = torch.where(here, z.gather(1, at)[:, 0], 0)
        loss = lse + z_weight * lse * lse - target
        loss_tol = tol * (1 + 2 * z_weight * lse.abs()) + torch.where(here, E.gather(1, at)[:, 0], 0) + 2.0 ** -22 * (target.abs() + loss.abs() + z_weight * lse * lse)
        none = self.labels < 0
        return torch.where(none, 0, loss), torch.where(none, 0, loss_tol), lse, tol

    def check_loss(self, z_weight=0.0, flags=0):
        loss, lse = self.loss(z_weight, flags)
        want, tol, want_lse, tol_lse = self.expected_loss(z_weight, 10 if flags else 20)
        assert bool(((lse.double() - want_lse).abs() <= tol_lse).all()), (lse.double() - want_lse).abs().div(tol_lse).max()
        assert bool(((loss.double() - want).abs() <= tol).all()), (loss.double() - want).abs().max()

    def gradient(self, out, lse, dloss, z_weight=0.0, sD=None, amax=None, flags=0, shift=0, stream=None):
        D = Guarded((self.M, self.N), DTYPE[out], shift)
        fp8.fp8_gemm_xent_grad(self.A, self.fa, self.tA, self.B, self.fb, self.tB, D.t, out, self.sA, self.sB, self.labels, lse, dloss, self.first, z_weight, sD, amax, flags, stream)
        D.check()
        return D.t

    def expected_gradient(self, lse, dloss, z_weight=0.0, bits=20):
        z, lse, d = self.z, lse.double()[:, None], dloss.double().expand(self.M)[:, None]
        p = torch.exp(z - lse) * (1 + 2 * z_weight * lse)
        hot = (torch.arange(self.N, device="cuda") + self.first)[None, :] == self.labels[:, None]
        y = d * (p - hot.double())
        tol = (d * p).abs() * torch.expm1(2.0 ** -bits * self.sizes + 2.0 ** -22 * (z.abs() + lse.abs() + 4)) + 2.0 ** -23 * d.abs() * hot + 1e-36
        none = (self.labels < 0)[:, None]
        return torch.where(none, 0, y), torch.where(none, 0, tol)

    def check_gradient(self, out, each=False, z_weight=0.0, sD=None, flags=0, shift=0, amax=True):
        lse = torch.logsumexp(self.z, 1).float()
        dloss = torch.linspace(0.25, 1.5, self.M, device="cuda") if each else torch.full((1,), 0.125, device="cuda")
        cell = torch.full((1,), 7.0, device="cuda") if amax else None
        D = self.gradient(out, lse, dloss, z_weight, sD, cell, flags, shift)
        y, tol = self.expected_gradient(lse, dloss, z_weight, 10 if flags else 20)
        if out in (O43, O52):
            fmt = E4M3 if out == O43 else E5M2
            most, tiny = (448.0, 2.0 ** -10) if out == O43 else (57344.0, 2.0 ** -17)
            s = 1.0 if sD is None else float(sD)
            got, y8, tol8 = D.view(TORCH8[fmt]).double(), (y * s).clamp(-most, most), tol * s
            half = torch.maximum((y8.abs() + tol8) * (2.0 ** -4 if out == O43 else 2.0 ** -3), torch.full_like(y8, tiny))
            assert bool(((got - y8).abs() <= tol8 + half + 2.0 ** -23 * y8.abs()).all())
        else:
            got = D.double()
            half = y.abs() * (2.0 ** -8 if out == BF16 else 2.0 ** -24)
            assert bool(((got - y).abs() <= tol * 1.01 + half).all()), ((got - y).abs() / (tol + half).clamp(min=1e-36)).max()
        assert bool((got[self.labels < 0] == 0).all())
        if amax:
            assert abs(float(cell) - float(y.abs().max())) <= float(tol.max()) + 2.0 ** -23 * float(y.abs().max())


# ---- shapes, forms, types -----------------------------------------------------------------------------------------------
SHAPES = [(1, 1, 16), (1, 50, 64), (3, 257, 33), (5, 1000, 1), (33, 130, 200), (64, 64, 128), (130, 515, 144), (300, 1003, 256), (257, 2049, 400)]


@pytest.mark.parametrize("name", FORMS)
@pytest.mark.parametrize("shape", SHAPES)
def test_loss_in_every_form(shape, name):
    with form(name):
        Problem(*shape).check_loss()
        Problem(*shape, seed=1, first=shape[1]).check_loss(z_weight=1e-2)


@pytest.mark.parametrize("name", FORMS)
@pytest.mark.parametrize("shape", SHAPES)
def test_gradient_in_every_form(shape, name):
    with form(name):
        Problem(*shape, seed=2).check_gradient(F32)
        Problem(*shape, seed=3, first=shape[1]).check_gradient(BF16, each=True, z_weight=1e-2)
        Problem(*shape, seed=4).check_gradient(O52, sD=torch.full((1,), 1000.0, device="cuda"))


@pytest.mark.parametrize("name", FORMS)
@pytest.mark.parametrize("tA,tB", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("shape", [(256, 512, 128), (304, 800, 192), (77, 333, 61)])
def test_storage_orders(shape, tA, tB, name):
    with form(name):
        p = Problem(*shape, tA=tA, tB=tB, seed=5)
        p.check_loss()
        p.check_gradient(F32, each=True)


@pytest.mark.parametrize("name", ["chosen", "fma", "small_32x64", "tiled_256"])
@pytest.mark.parametrize("fa,fb", [(E4M3, E5M2), (E5M2, E4M3), (E5M2, E5M2)])
def test_formats(fa, fb, name):
    with form(name):
        p = Problem(200, 700, 96, fa=fa, fb=fb, seed=6)
        p.check_loss()
        p.check_gradient(O52)


@pytest.mark.parametrize("name", FORMS)
@pytest.mark.parametrize("rows,columns", [(True, False), (False, True), (True, True)])
@pytest.mark.parametrize("shape", [(7, 129, 80), (270, 900, 128)])
def test_factors(shape, rows, columns, name):
    with form(name):
        p = Problem(*shape, rows=rows, columns=columns, seed=7)
        p.check_loss(z_weight=1e-3)
        p.check_gradient(F32, each=True, z_weight=1e-3)


@pytest.mark.parametrize("name", ["chosen", "tiled_128", "tiled_256", "tiled_both"])
@pytest.mark.parametrize("out,shift", [(F32, 1), (F32, 0), (BF16, 3), (O43, 0), (O43, 5), (O52, 1)])
@pytest.mark.parametrize("N", [512, 515])
def test_outputs_at_any_element(out, shift, name, N):
    with form(name):
        Problem(260, N, 128, seed=8).check_gradient(out, shift=shift, sD=torch.full((1,), 300.0, device="cuda") if out in (O43, O52) else None)


@pytest.mark.parametrize("shift", [1, 7, 8])
def test_operands_at_any_byte(shift):
    p = Problem(130, 300, 96, seed=9, shift=shift)
    p.check_loss()
    p.check_gradient(BF16)


@pytest.mark.parametrize("name", ["chosen", "small_32x32", "small_64x64", "tiled_128", "tiled_256", "tiled_both"])
@pytest.mark.parametrize("shape", [(5, 300, 128), (300, 1100, 256), (100, 333, 129)])
def test_fp8_instructions(shape, name):
    with form(name):
        p = Problem(*shape, seed=10)
        p.check_loss(flags=fp8.FP8_GEMM_MFMA8)
        p.check_gradient(BF16, flags=fp8.FP8_GEMM_MFMA8)


# ---- empty and degenerate -------------------------------------------------------------------------------------------------
def test_no_rows_no_columns_no_inner_dimension():
    p = Problem(0, 10, 16)
    p.loss()
    p = Problem(4, 0, 16)
    p.labels = torch.tensor([0, -1, 3, 0], device="cuda")
    loss, lse = p.loss()
    assert lse.tolist() == [-math.inf] * 4 and loss.tolist() == [-math.inf, 0.0, -math.inf, -math.inf]
    cell = torch.full((1,), 3.0, device="cuda")
    p.gradient(F32, lse, torch.ones(1, device="cuda"), amax=cell)
    assert float(cell) == 0.0
    p = Problem(6, 100, 0)
    p.check_loss()
    p.check_gradient(F32)


@pytest.mark.parametrize("name", FORMS)
def test_no_row_has_a_label(name):
    with form(name):
        p = Problem(260, 300, 64, seed=11)
        p.labels.fill_(-1)
        loss, lse = p.loss(z_weight=0.1)
        assert bool((loss == 0).all()) and bool(torch.isfinite(lse).all())
        cell = torch.full((1,), 3.0, device="cuda")
        D = p.gradient(F32, lse, torch.ones(1, device="cuda"), amax=cell)
        assert bool((D == 0).all()) and float(cell) == 0.0


@pytest.mark.parametrize("name", FORMS)
def test_infinities_and_nan(name):
    """Operands in E5M2 hold infinities; the tokens have a 1 in one place each, so that a logit is an element of the weight."""
    inf, nan = math.inf, math.nan
    M, N, K = 8, 300, 16
    with form(name):
        p = Problem(M, N, K, fa=E5M2, fb=E5M2, seed=12)
        p.sA.fill_(1.0)
        p.sB.fill_(1.0)
        a = torch.zeros(M, K, device="cuda")
        b = torch.randn(N, K, device="cuda")
        for i in range(M):
            a[i, i] = 1.0
        # (the other places of a row of the weight are multiplied by 0: an infinity there would be NaN)
        p.set(a.to(torch.float8_e5m2), b.to(torch.float8_e5m2))
        z = p.z.clone()
        loss, lse = p.loss()
        assert torch.allclose(lse.double(), torch.logsumexp(z, 1), atol=1e-5)
        for value, row_lse in ((-inf, None), (inf, inf), (nan, nan)):
            # one token, so that no other row sees the value
            q = Problem(1, N, 1, fa=E5M2, fb=E5M2, seed=13)
            q.sA.fill_(1.0)
            q.sB.fill_(1.0)
            w = torch.randn(N, 1, device="cuda")
            w[5] = w[290] = value
            q.set(torch.ones(1, 1, device="cuda").to(torch.float8_e5m2), w.to(torch.float8_e5m2))
            q.labels[:] = 7
            loss, lse = q.loss()
            want = torch.logsumexp(q.z, 1)
            if value == -inf:
                assert torch.allclose(lse.double(), want, atol=1e-5)
                D = q.gradient(F32, lse, torch.ones(1, device="cuda"))
                assert float(D[0, 5]) == 0.0 and float(D[0, 290]) == 0.0 and bool(torch.isfinite(D).all())
                q.labels[:] = 5
                assert q.loss()[0].item() == inf
            else:
                assert lse.item() == row_lse or math.isnan(row_lse) and math.isnan(lse.item())
            # without a label nothing of it is seen
            q.labels[:] = -5
            loss, lse = q.loss(z_weight=0.5)
            D = q.gradient(F32, lse, torch.ones(1, device="cuda"), z_weight=0.5)
            assert loss.item() == 0.0 and bool((D == 0).all())
        # nothing but -infinity
        q.set(torch.ones(1, 1, device="cuda").to(torch.float8_e5m2), torch.full((N, 1), -inf, device="cuda").to(torch.float8_e5m2))
        assert q.loss()[1].item() == -inf


@pytest.mark.parametrize("name", FORMS)
def test_nan_in_e4m3_operands(name):
    """A token of NaN (its rows: NaN, but 0 without a label) and a NaN in the weight (a column of every row)."""
    with form(name):
        p = Problem(270, 600, 64, seed=27)
        p.labels[5], p.labels[6], p.labels[200] = 17, -1, -1
        p.A[5, 3] = p.A[6, 63] = p.A[200, 0] = 0x7F
        loss, lse = p.loss()
        bad = torch.zeros(270, dtype=torch.bool, device="cuda")
        bad[[5, 6, 200]] = True
        assert bool(torch.isnan(lse[bad]).all()) and math.isnan(float(loss[5])) and float(loss[6]) == float(loss[200]) == 0.0
        want, tol, want_lse, tol_lse = p.expected_loss()
        assert bool(((lse.double() - want_lse).abs() <= tol_lse)[~bad].all()) and bool(((loss.double() - want).abs() <= tol)[~bad].all())
        one = torch.ones(1, device="cuda")
        for out in (F32, BF16, O52):
            D = p.gradient(out, lse, one)
            D = D.view(torch.float8_e5m2).float() if out == O52 else D.float()
            assert bool(torch.isnan(D[5]).all()) and bool((D[p.labels < 0] == 0).all()) and bool(torch.isfinite(D[~bad]).all())
        p = Problem(270, 600, 64, seed=28)
        good = p.loss()[1].clone()
        p.B[599, 8] = 0xFF
        loss, lse = p.loss(z_weight=1e-2)
        assert bool(torch.isnan(lse).all()) and bool((loss[p.labels < 0] == 0).all()) and bool(torch.isnan(loss[p.labels >= 0]).all())
        D = p.gradient(F32, good, one)
        assert bool((D[p.labels < 0] == 0).all()) and bool(torch.isnan(D[p.labels >= 0][:, 599]).all()) and bool(torch.isfinite(D[:, :599]).all())


@pytest.mark.parametrize("name", FORMS)
def test_factors_of_the_output_below_one(name):
    with form(name):
        for each in (False, True):
            Problem(270, 700, 64, seed=30, rows=each).check_gradient(O43, each=each, sD=torch.full((1,), 0.25, device="cuda"))


@pytest.mark.parametrize("name", FORMS)
@pytest.mark.parametrize("sD,dloss", [(0.0, 1.0), (math.inf, 1.0), (math.nan, 1.0), (2.0 ** -140, 1.0), (2.0 ** -60, 1.0), (2.0 ** 126, 8.0), (-(2.0 ** 126), 8.0), (2.0 ** 100, 2.0 ** 29), (2.0 ** -20, 2.0 ** 30)])
def test_factors_of_the_output_far_from_one(name, sD, dloss):
    """All of a piece's probabilities are 2^-96 of a softmax, as of rows whose label is in another piece: dloss sD of 2^129, beyond fp32, where outputs are inside E5M2;
    outputs that vanish beside a maximum that does not; factors of 0, infinity and NaN.  y is off by what check_gradient counts, its product with sD rounds once more."""
    M, N, K = 260, 300, 32
    with form(name):
        p = Problem(M, N, K, seed=29, first=1000)
        p.labels.fill_(3)
        p.labels[7] = -1
        lse = (torch.logsumexp(p.z, 1) + 96.0 * math.log(2.0)).float()
        d, cell, s = torch.full((1,), dloss, device="cuda"), torch.full((1,), 7.0, device="cuda"), torch.full((1,), sD, device="cuda")
        for amax in (cell, None):
            D = p.gradient(O52, lse, d, 0.0, s, amax).view(torch.float8_e5m2).double()
            y, tol = p.expected_gradient(lse, d)
            # what underflows: an exponential below the smallest normal number, 2^-126, is 0 (a logit 20.8 below its row's sum is): dloss 2^-126 in place of 1e-36
            tol = tol + torch.where(p.labels < 0, 0, dloss * 2.0 ** -126 - 1e-36)[:, None]
            if math.isfinite(sD):
                y8, tol8 = (y * sD).clamp(-57344, 57344), tol * abs(sD)
                half = torch.maximum((y8.abs() + tol8) * 2.0 ** -3, torch.full_like(y8, 2.0 ** -17))
                assert bool(((D - y8).abs() <= tol8 + half + 2.0 ** -23 * y8.abs()).all())
            elif math.isnan(sD):
                assert bool(torch.isnan(D[p.labels >= 0]).all())
            else:
                full = y >= 2.0 ** -125                                              # (y infinity is one, which E5M2 holds; 0 infinity is none)
                assert bool((D[full] == math.inf).all()) and int(full.sum()) > 0.99 * 259 * N and not bool(torch.isfinite(D[p.labels >= 0]).any())
        assert abs(float(cell) - float(y.max())) <= float(tol.max()) + 2.0 ** -23 * float(y.max())


@pytest.mark.parametrize("name", FORMS)
def test_negative_factors(name):
    with form(name):
        p = Problem(300, 600, 128, seed=29)
        p.sA.neg_()
        p.z = -p.z
        p.check_loss(z_weight=1e-3)
        p.check_gradient(F32, each=True)


@pytest.mark.parametrize("name", ["chosen", "fma", "small_32x64", "tiled_256", "tiled_128"])
@pytest.mark.parametrize("spread", [1e-3, 60.0, 3000.0])
def test_flat_and_peaked_rows(name, spread):
    with form(name):
        p = Problem(100, 1000, 128, spread=spread, seed=14)
        p.check_loss()
        p.check_gradient(F32)


def test_the_formulas_against_differences():
    """expected_gradient, which everything above is compared with, against differences of expected_loss in 64 bits."""
    p = Problem(9, 40, 16, seed=15, first=3)
    w, h = 0.02, 1e-6
    lse = torch.logsumexp(p.z, 1)
    y, _ = p.expected_gradient(lse, torch.ones(1, device="cuda"), w)
    z = p.z.clone()
    for j in range(p.N):
        p.z = z.clone(); p.z[:, j] += h
        up = p.expected_loss(w)[0]
        p.z = z.clone(); p.z[:, j] -= h
        down = p.expected_loss(w)[0]
        # second differences of the loss are below 4, third ones below 8: h^2 8 / 6; loss values of up to 10 round at 2^-53
        assert bool((((up - down) / (2 * h) - y[:, j]).abs() < 2 * h * h + 20 * 2.0 ** -53 / h).all())


# ---- pieces of a vocabulary ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("sizes", [(400, 400, 203), (1, 1001, 1)])
def test_a_vocabulary_in_pieces(sizes):
    whole = Problem(150, sum(sizes), 128, seed=16)
    whole.labels[0] = sizes[0]
    loss, lse = whole.loss()
    dloss = torch.full((1,), 0.01, device="cuda")
    D = whole.gradient(F32, lse, dloss)
    first, parts, pieces = 0, [], []
    for n in sizes:
        p = Problem.__new__(Problem)
        p.__dict__.update(whole.__dict__)
        p.N, p.first, p.B = n, first, whole.B[first:first + n].contiguous()
        parts.append(p.loss())
        pieces.append(p.gradient(F32, lse, dloss))
        first += n
    total = torch.logsumexp(torch.stack([x[1].double() for x in parts]), 0)
    joined = torch.where(whole.labels < 0, 0, total + sum(x[0].double() - torch.where(whole.labels < 0, 0, x[1].double()) for x in parts))
    want, tol, want_lse, tol_lse = whole.expected_loss()
    assert bool(((total - want_lse).abs() <= 2 * tol_lse).all()) and bool(((joined - want).abs() <= 2 * tol + 4 * tol_lse).all())
    y, tol = whole.expected_gradient(lse, dloss)
    assert bool(((torch.cat(pieces, 1).double() - y).abs() <= 1.01 * tol).all()) and bool(((D.double() - y).abs() <= 1.01 * tol).all())


# ---- sizes beyond 32 bits -------------------------------------------------------------------------------------------------
def test_an_output_of_more_than_2_32_bytes():
    M, N, K = 70000, 65537, 16
    g = torch.Generator(device="cuda").manual_seed(17)
    a8 = torch.randn((M, K), generator=g, device="cuda").to(torch.float8_e4m3fn)
    b8 = torch.randn((N, K), generator=g, device="cuda").to(torch.float8_e4m3fn)
    one = torch.ones(1, device="cuda")
    labels = torch.randint(0, N, (M,), generator=g, device="cuda")
    loss, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    ws = torch.empty(fp8.fp8_gemm_xent_workspace_size(M, N), dtype=torch.uint8, device="cuda")
    A, B = a8.view(torch.uint8), b8.view(torch.uint8)
    fp8.fp8_gemm_xent(A, E4M3, False, B, E4M3, True, labels, loss, lse, ws, one, one)
    D = torch.empty((M, N), dtype=torch.uint8, device="cuda")
    sD = torch.full((1,), 16384.0, device="cuda")
    fp8.fp8_gemm_xent_grad(A, E4M3, False, B, E4M3, True, D, O52, one, one, labels, lse, one, sD=sD)
    for at in (0, 33333, 65535, M - 64):
        rows = slice(at, at + 64)
        z = a8[rows].double() @ b8.double().t().contiguous()
        E = 2.0 ** -20 * (a8[rows].double().abs() @ b8.double().abs().t().contiguous())
        want = torch.logsumexp(z, 1)
        tol = E.amax(1) + 2.0 ** -22 * (want.abs() + z.abs().amax(1)) + 2.0 ** -19
        assert bool(((lse[rows].double() - want).abs() <= tol).all())
        here = torch.arange(64, device="cuda"), labels[rows]
        assert bool(((loss[rows].double() - want + z[here]).abs() <= tol + E[here] + 2.0 ** -21 * (z[here].abs() + want.abs())).all())
        l = lse[rows].double()[:, None]
        p = torch.exp(z - l)
        y = p.clone()
        y[here] -= 1
        y *= 16384.0
        tol = 16384.0 * (p * torch.expm1(E + 2.0 ** -22 * (z.abs() + l.abs() + 4)) + 2.0 ** -23)
        got = D[rows].view(torch.float8_e5m2).double()
        assert bool(((got - y).abs() <= tol + torch.clamp((y.abs() + tol) * 2.0 ** -3, min=2.0 ** -17)).all())


def test_a_workspace_of_more_than_2_32_bytes():
    M, N, K = 1 << 19, 40000, 16
    g = torch.Generator(device="cuda").manual_seed(18)
    a8 = torch.randn((M, K), generator=g, device="cuda").to(torch.float8_e4m3fn)
    b8 = torch.randn((N, K), generator=g, device="cuda").to(torch.float8_e4m3fn)
    one = torch.ones(1, device="cuda")
    labels = torch.randint(0, N, (M,), generator=g, device="cuda")
    loss, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    size = fp8.fp8_gemm_xent_workspace_size(M, N)
    assert size > 1 << 32
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    for name in ("chosen", "small_64x64"):
        print(name)
        with form(name):
            fp8.fp8_gemm_xent(a8.view(torch.uint8), E4M3, False, b8.view(torch.uint8), E4M3, True, labels, loss.fill_(0), lse.fill_(0), ws, one, one)
        for at in (0, M - 100):
            rows = slice(at, at + 100)
            z = a8[rows].double() @ b8.double().t().contiguous()
            want = torch.logsumexp(z, 1)
            tol = 2.0 ** -20 * (a8[rows].double().abs() @ b8.double().abs().t().contiguous()).amax(1) + 2.0 ** -22 * (want.abs() + z.abs().amax(1)) + 2.0 ** -19
            assert bool(((lse[rows].double() - want).abs() <= tol).all())
            assert bool(((loss[rows].double() - want + z.gather(1, labels[rows][:, None])[:, 0]).abs() <= 2 * tol + 2.0 ** -20 * want.abs()).all())
    # 1.05 10^10 threads, more than a launch has: refused, not left undone
    with form("small_32x32"), pytest.raises(fp8.Fp8Error, match="grid limit"):
        fp8.fp8_gemm_xent(a8.view(torch.uint8), E4M3, False, b8.view(torch.uint8), E4M3, True, labels, loss, lse, ws, one, one)


# ---- runs, streams, graphs ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("shape", [(1, 5000, 256), (300, 5000, 256), (1000, 2000, 128)])
def test_the_same_in_every_run(shape):
    p = Problem(*shape, seed=19)
    first = [x.clone() for x in p.loss()]
    dloss = torch.ones(1, device="cuda")
    D = p.gradient(BF16, first[1], dloss).clone()
    junk = torch.empty(1 << 26, device="cuda")
    for _ in range(5):
        junk.normal_()
        again = p.loss()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
        assert torch.equal(D, p.gradient(BF16, first[1], dloss))


def test_on_another_stream_and_two_at_once():
    ps = [Problem(200, 3000, 128, seed=20), Problem(333, 2000, 256, seed=21)]
    dloss = torch.ones(1, device="cuda")
    want = []
    for p in ps:
        loss, lse = p.loss()
        want.append((loss.clone(), lse.clone(), p.gradient(BF16, lse, dloss).clone()))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    kept = [[torch.empty_like(x) for x in w] for w in want]
    spaces = [torch.empty(fp8.fp8_gemm_xent_workspace_size(p.M, p.N), dtype=torch.uint8, device="cuda") for p in ps]
    torch.cuda.synchronize()
    for _ in range(10):
        for p, s, (loss, lse, D), ws in zip(ps, streams, kept, spaces):
            fp8.fp8_gemm_xent(p.A, p.fa, p.tA, p.B, p.fb, p.tB, p.labels, loss, lse, ws, p.sA, p.sB, stream=s)
            fp8.fp8_gemm_xent_grad(p.A, p.fa, p.tA, p.B, p.fb, p.tB, D, BF16, p.sA, p.sB, p.labels, lse, dloss, stream=s)
    torch.cuda.synchronize()
    for w, k in zip(want, kept):
        assert all(torch.equal(x, y) for x, y in zip(w, k))


def test_captured_and_replayed():
    p = Problem(300, 3001, 128, seed=22)
    loss, lse = torch.zeros(p.M, device="cuda"), torch.zeros(p.M, device="cuda")
    ws = torch.empty(fp8.fp8_gemm_xent_workspace_size(p.M, p.N), dtype=torch.uint8, device="cuda")
    D, dloss, amax = torch.zeros((p.M, p.N), dtype=torch.uint8, device="cuda"), torch.ones(1, device="cuda"), torch.zeros(1, device="cuda")

    def step():
        fp8.fp8_gemm_xent(p.A, p.fa, p.tA, p.B, p.fb, p.tB, p.labels, loss, lse, ws, p.sA, p.sB, z_weight=1e-3)
        fp8.fp8_gemm_xent_grad(p.A, p.fa, p.tA, p.B, p.fb, p.tB, D, O52, p.sA, p.sB, p.labels, lse, dloss, z_weight=1e-3, amax_out=amax)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (23, 24, 25):
        q = Problem(300, 3001, 128, seed=seed)
        for mine, other in ((p.A, q.A), (p.B, q.B), (p.labels, q.labels), (p.sA, q.sA), (p.sB, q.sB)):
            mine.copy_(other)
        step()
        torch.cuda.synchronize()
        want = [x.clone() for x in (loss, lse, D, amax)]
        for x in (loss, lse, D, amax):
            x.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, (loss, lse, D, amax)))


# ---- the Python binding -------------------------------------------------------------------------------------------------
def test_refusals_of_the_binding():
    p = Problem(8, 40, 16, seed=26)
    loss, lse = torch.empty(8, device="cuda"), torch.empty(8, device="cuda")
    ws, one = torch.empty(4096, dtype=torch.uint8, device="cuda"), torch.ones(1, device="cuda")
    D = torch.empty((8, 40), device="cuda")

    def forward(labels=p.labels, loss=loss, lse=lse, ws=ws, B=p.B):
        fp8.fp8_gemm_xent(p.A, E4M3, False, B, E4M3, True, labels, loss, lse, ws, p.sA, p.sB)

    def backward(labels=p.labels, lse=lse, dloss=one, D=D):
        fp8.fp8_gemm_xent_grad(p.A, E4M3, False, p.B, E4M3, True, D, F32, p.sA, p.sB, labels, lse, dloss)
    forward(), backward()
    for wrong in (dict(labels=p.labels.int()), dict(labels=p.labels[:7]), dict(labels=p.labels.cpu()), dict(lse=lse[:7]), dict(lse=lse.double())):
        for call in (forward, backward):
            with pytest.raises(ValueError):
                call(**wrong)
    for wrong in (dict(loss=loss[:7]), dict(B=p.B[:, :8])):
        with pytest.raises(ValueError):
            forward(**wrong)
    with pytest.raises(ValueError):
        backward(D=D[:, :30])
    with pytest.raises(fp8.Fp8Error):
        forward(ws=ws[:100])
    with pytest.raises(fp8.Fp8Error):
        backward(dloss=torch.ones(3, device="cuda"))
