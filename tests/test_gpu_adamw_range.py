"""AdamW to the last bit, and where its numbers leave the ordinary range: second moments below the smallest normal number, with eps = 0 too, factors whose
reciprocal lies there, denominators that have no normal reciprocal.

Tolerances as in test_gpu_adamw.py, u = 2^-24; below 2^-126 every rounding is off by up to 2^-150 instead: v' has at most five (the square of sqrt(v) as stored, two products of the
gradient's square, b2 v, the sum), and is off by 16u v' + 5 2^-150."""
import math

import pytest
import torch

import paper_2209_05433_amd as fp8

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STEP0 = 5 * 2.0 ** -150
F8 = torch.float8_e4m3fn
BLOCK = fp8.FP8_STATE_BLOCK


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


def blocks_of(tops, gen):
    """Codes of blocks with elements of all sizes, and the factors that make their largest `tops`."""
    codes = (torch.rand(len(tops), BLOCK, generator=gen, device="cuda") * 447).to(F8)
    codes[:, 3] = 448.0
    return codes.view(torch.uint8).view(-1), (448.0 / torch.tensor(tops, dtype=torch.float64)).float().cuda()


# (of r: v' from above 2^-126 down to some units of 2^-149)
TOPS = [2.0 ** -62, 1.3 * 2.0 ** -63, 1.1e-19, 2.0 ** -65, 3e-20, 2.0 ** -68, 1e-21, 2e-22, 2.0 ** -73]


@pytest.mark.parametrize("g", [0.0, 1e-19, 1e-5])
def test_second_moments_below_the_normal_numbers(g):
    """One step from sqrt(v) of about 1e-19, gradients in one half of each block or in none."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    v, vs = blocks_of(TOPS, gen)
    n = v.numel()
    r0 = v.view(F8).double() / vs.double().repeat_interleave(BLOCK)
    m, ms, p = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.ones(len(TOPS), device="cuda"), torch.zeros(n, device="cuda")
    grad = torch.zeros(n, device="cuda")
    grad.view(-1, BLOCK)[:, 64:] = g
    fp8.fp8_adamw([p], [grad], [m], [v], cells(2000, torch.int64), cells(1e-2), 0.9, 0.95, m_scale=[ms], v_scale=[vs], seed=5)
    want_v = 0.95 * r0 * r0 + (1 - 0.95) * grad.double().square()
    tol_v = 16 * U * want_v + STEP0
    low, want, high = ((want_v + d).clamp(min=0).sqrt() for d in (-tol_v, 0, tol_v))
    # the block's factor is 448 over the largest, the largest's code 448 (or the one below, by one random number in 2^16)
    top_low, top, top_high = (x.view(-1, BLOCK).amax(1) for x in (low, want, high))
    assert bool((vs.double() >= 448 / top_high * (1 - 4 * U)).all()) and bool((vs.double() <= 448 / top_low * (1 + 4 * U)).all()), (vs.double() * top / 448)
    got = v.view(F8).double()
    scale = vs.double().repeat_interleave(BLOCK)
    a = (want * scale).clamp(max=448.0)
    slack = torch.maximum(high - want, want - low) * scale + 4 * U * a
    gap = torch.exp2((torch.floor(torch.log2((a + slack).clamp(min=2.0 ** -30))) - 3).clamp(min=-9))
    assert bool(((got - a).abs() <= gap + slack).all())
    assert bool((got[want_v > 2 * STEP0] > 0).all())


@pytest.mark.parametrize("beta2", [0.95, 0.5])
def test_a_block_without_gradients_decays(beta2):
    """Step after step, past 2^-126 of v: sqrt(v) of the largest goes down by sqrt(beta2) (to the units of 2^-149 where beta2 v rounds to v), and what is smaller stays so."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    v, vs = blocks_of([1e-3, 1e-3, 0.7e-3], gen)
    n = v.numel()
    m, ms, p, g = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.ones(3, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    steps = int(2 * math.log(1e-3 / 2.0 ** -74) / -math.log(beta2)) + 50
    for t in range(1, steps + 1):
        fp8.fp8_adamw([p], [g], [m], [v], cells(t, torch.int64), cells(1e-2), 0.9, beta2, m_scale=[ms], v_scale=[vs], seed=6)
        if t % 10 == 0 or t > steps - 300:
            r = (v.view(F8).double() / vs.double().repeat_interleave(BLOCK)).view(-1, BLOCK).amax(1)
            # (a step: factor and read two roundings each, root one, square, product and beta2 a half each; a unit of 2^-149 in which v is rounded a step, 1 / (1 - beta2) together)
            most = 1e-3 * beta2 ** (t / 2) * (1 + 8 * U * t) + math.sqrt(2.0 ** -149 / (1 - beta2))
            assert bool((r <= most).all()), (t, r.tolist(), most)
    # the next gradient counts for what it is: p moves by lr times 0.1 / (1 - 0.9^t) over sqrt((1 - beta2) / (1 - beta2^t))
    g.fill_(1e-5)
    fp8.fp8_adamw([p], [g], [m], [v], cells(steps + 1, torch.int64), cells(1e-2), 0.9, beta2, 0.0, m_scale=[ms], v_scale=[vs], seed=6)
    want = -1e-2 * 0.1 / math.sqrt(1 - beta2)
    assert bool(((p.double() - want).abs() <= 64 * U * abs(want) + abs(want) * 0.9 ** steps).all())


@pytest.mark.parametrize("p_dtype", [torch.float32, torch.bfloat16])
def test_states_in_32_bits_without_eps(p_dtype):
    """v' from 2^-120 down to 2^-148, eps = 0: the weights move by what the formula says.  v' is off by 16u v' + 5 2^-150, the update by what that makes of it and 32u."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    n = 5000
    v = torch.exp2(-120 - 28 * torch.rand(n, generator=gen, device="cuda").double()).float()
    m = torch.randn(n, generator=gen, device="cuda") * v.double().sqrt().float()
    g = torch.zeros(n, device="cuda")
    g[::2] = (v[::2].double().sqrt() * 3).float()
    p = torch.ones(n, device="cuda").to(p_dtype)
    m0, v0, g0 = m.double(), v.double(), g.double()
    fp8.fp8_adamw([p], [g], [m], [v], cells(7, torch.int64), cells(1e-2), 0.9, 0.95, 0.0)
    m1, v1 = 0.9 * m0 + (1 - 0.9) * g0, 0.95 * v0 + (1 - 0.95) * g0 * g0
    m_tol, v_tol = 16 * U * ((0.9 * m0).abs() + ((1 - 0.9) * g0).abs()) + STEP0, 16 * U * v1 + STEP0
    assert bool(((m.double() - m1).abs() <= m_tol).all()) and bool(((v.double() - v1).abs() <= v_tol).all())
    k1, k2 = 1 / (1 - 0.9 ** 7), (1 - 0.95 ** 7) ** 0.5
    u = 1e-2 * k1 * k2 * m1 / v1.sqrt()
    far = 1e-2 * k1 * k2 * ((m1.abs() + m_tol) / (v1 - v_tol).clamp(min=2.0 ** -150).sqrt() - m1.abs() / v1.sqrt())
    want = 1.0 - u
    tol = far + 32 * U * u.abs() + U * want.abs() + (2.0 ** -8 * want.abs() if p_dtype == torch.bfloat16 else 0)
    assert bool(torch.isfinite(p).all()) and bool(((p.double() - want).abs() <= tol * 1.01).all()), ((p.double() - want).abs() / tol).max()


@pytest.mark.parametrize("which", ["m", "v"])
def test_factors_whose_reciprocal_is_not_normal(which):
    """m = byte / factor for every finite factor > 0, 2^127 and 3e38 among them, and the smallest; elements of 0 beside."""
    factors = torch.tensor([2.0 ** 126, 1.5 * 2.0 ** 126, 2.0 ** 127, 3e38, 2.0 ** -126, 2.0 ** -127, 2.0 ** -120], device="cuda")
    n = len(factors) * BLOCK
    codes = torch.zeros(n, device="cuda")
    codes.view(-1, BLOCK)[:, ::3] = 1.0
    codes.view(-1, BLOCK)[:, 1] = 448.0 if which == "m" else 2.0
    codes = codes.to(F8)
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    zero, one = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.ones(len(factors), device="cuda")
    state, scale = codes.view(torch.uint8).clone(), factors.clone()
    m, ms, v, vs = (state, scale, zero, one) if which == "m" else (zero, one, state, scale)
    x0 = codes.double() / factors.double().repeat_interleave(BLOCK)
    # eps of 1: with v = 0 the weights move by lr m' / (1 - beta1^t) = 2 m'; a reciprocal below 2^-126 is off by up to 2^-22 of itself, 4u
    fp8.fp8_adamw([p], [g], [m], [v], cells(1, torch.int64), cells(1.0), 0.5, 0.25, 1.0, m_scale=[ms], v_scale=[vs], seed=7)
    if which == "m":
        x1 = 0.5 * x0
        fine = x0 < 3e38              # (beyond: 448 2^120 = 6e38, which is m and the step of p, is no number in 32 bits)
        assert bool(((p.double() + 2 * x1)[fine].abs() <= 32 * U * x1[fine] + 4 * STEP0).all()), (p.double().view(-1, BLOCK)[:, 1], x1.view(-1, BLOCK)[:, 1])
    else:
        # (v' of factors this large is 0; of the smallest ones it is infinite, and r with it)
        x1 = 0.5 * x0
        x1 = torch.where(x0 * x0 < 2.0 ** -150, torch.zeros_like(x1), x1)
        fine = x0 * x0 < 3e38
        assert not bool(p.any())
    got = state.view(F8).double() / scale.double().repeat_interleave(BLOCK)
    top = x1.view(-1, BLOCK).amax(1, keepdim=True).expand(-1, BLOCK).reshape(-1)
    # (a block whose factor would not be finite: factor 1, where these are rounded to 0)
    kept = 448.0 / top.clamp(min=1e-300) < 3.4e38
    want = torch.where(kept, x1, torch.zeros_like(x1))
    inside = fine.view(-1, BLOCK).all(1).repeat_interleave(BLOCK)
    assert bool(((got - want).abs()[inside] <= 2.0 ** -3 * want[inside] + 2.0 ** -9 / 448 * top[inside] * kept[inside]).all())
    assert bool((scale.double().repeat_interleave(BLOCK)[inside & ~kept] == 1).all()) and bool((scale[4:] > 0).all())


@pytest.mark.parametrize("states8", [False, True])
@pytest.mark.parametrize("eps,m0", [(1e-40, 2.0 ** -136), (2e-38, 2.0 ** -120), (2.5e38, 1e38), (2.0 ** 127, 2.0 ** 125), (1e-30, 1e-30)])
def test_denominators_without_a_normal_reciprocal(states8, eps, m0):
    """v = 0: the update is lr (m' / (1 - beta1^t)) / eps.  1 - beta1^t is 3/4; eps times it is off by 2^-24 of itself or 2^-150."""
    n = 300
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    if states8:
        m, v = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
        factor = min(256.0 / m0, 2.0 ** 127)
        code = torch.tensor([m0 * factor], dtype=torch.float64).float().to(F8)
        m0 = float(code.double()) / float(torch.tensor(factor).float())
        m.fill_(int(code.view(torch.uint8)))
        more = dict(m_scale=[torch.full((3,), factor, device="cuda")], v_scale=[torch.ones(3, device="cuda")])
    else:
        m, v, more = torch.full((n,), m0, device="cuda"), torch.zeros(n, device="cuda"), {}
        m0 = float(m[0])
    fp8.fp8_adamw([p], [g], [m], [v], cells(2, torch.int64), cells(1e-2), 0.5, 0.5, eps, **more)
    e = float(torch.tensor(eps))
    want = -1e-2 * (0.5 * m0 / 0.75) / e
    tol = abs(want) * (32 * U + 2.0 ** -149 / (0.75 * e))
    assert bool(((p.double() - want).abs() <= tol).all()), (p[0].item(), want)
