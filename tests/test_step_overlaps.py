"""Memory that the gradient of the loss or AdamW writes and that is an argument otherwise too: refused on the host, nothing is launched."""
import random

import pytest

import paper_2209_05433_amd as fp8
from test_step_refusals import A, B, BAD, D, F, K, M, N, S, SCALES, W, Z, adamw, grad

# (the gradient of test_step_refusals: D of M x N bytes at D, factors at F, dloss at F + 64, labels at S, lse at Z)


@pytest.mark.parametrize("wrong", [
    dict(D=F - M * N + 1), dict(D=F), dict(sA=D + 4), dict(sB=D + M * N - 4), dict(sA=D + M * N - 4, nsA=M), dict(sA=D - 4 * M + 4, nsA=M), dict(sB=D - 4 * N + 4, nsB=N), dict(sD=D + 8), dict(amax=D),
    dict(amax=D + M * N - 4), dict(out_kind=0, amax=D + 4 * M * N - 4), dict(amax=A), dict(amax=A + M * K - 4), dict(amax=B + 4), dict(amax=S), dict(amax=S + 8 * M - 4), dict(amax=Z + 4 * M - 4)])
def test_the_gradient(wrong):
    assert grad(**wrong) == BAD and "overlap" in fp8.fp8_last_error(), fp8.fp8_last_error()


def test_an_output_of_nothing_overlaps_nothing():
    assert grad(N=0, D=S + 8) == fp8.FP8_OK and grad(M=0, ndloss=1, D=F + 64) == fp8.FP8_OK


# (AdamW of test_step_refusals: tensors of 200 and 3 elements, 4096 bytes apart: weights in fp32 and bf16 at A, gradients in bf16 and fp32 at B, states at D and D + 8192, lr at F, step at S;
# SCALES: states in FP8, factors at Z, Z + 64, Z + 128, Z + 192)
ADAM_F32 = [
    dict(g=(B, A)), dict(g=(A + 4096, B)), dict(g=(B, A + 796)), dict(g=(A - 398, B + 4096)), dict(m=(D, D + 8192 + 796)), dict(m=(D, D)),
    dict(v=(D + 8192, D + 8192)), dict(v=(D + 4096 + 8, D + 12288)), dict(m=(A + 4096, D + 4096)), dict(m=(D, B)), dict(v=(B + 4096, D)), dict(q=(A + 4096, None), q_scale=F), dict(q=(None, D + 799), q_scale=F),
    dict(q=(W, W + 199), q_scale=F), dict(q=(B + 4096 + 11, None), q_scale=F), dict(lr=A + 796), dict(lr=D), dict(step=D + 8192 + 792), dict(norm=A), dict(q=(W, None), q_scale=D),
    dict(q=(F + 1024 - 199, None), q_scale=F + 1024), dict(q=(W, None), q_scale=W + 196), dict(q_amax=A), dict(q_amax=D + 796), dict(q_amax=B + 396), dict(q_amax=B + 4096 - 4),
    dict(q=(W, None), q_scale=F, q_amax=W + 192), dict(lr=W + 196, q=(W, None), q_scale=F)]
ADAM_FP8 = [dict(m_scale=(Z, Z + 4)), dict(m_scale=(Z, Z + 132)), dict(v_scale=(Z + 128, Z + 64)), dict(v_scale=(A + 196, Z)), dict(m_scale=(D + 196, Z)), dict(m_scale=(Z, B + 4096)), dict(norm=Z + 64),
            dict(lr=Z + 132), dict(q_amax=Z + 124), dict(m=(D, D + 197)), dict(m=(Z - 199, D + 4096))]


@pytest.mark.parametrize("wrong", ADAM_F32 + [dict(SCALES, **x) for x in ADAM_FP8])
def test_adamw(wrong):
    assert adamw(**wrong) == BAD and "overlap" in fp8.fp8_last_error(), fp8.fp8_last_error()


@pytest.mark.parametrize("states8", [False, True])
def test_adamw_on_random_places(states8):
    """Up to 40 tensors anywhere in little memory, against every pair of ranges: refused if one of the two is written.  (Calls that are fine are made with a weight in the wrong place
    in the end, so that none is launched: a misaligned one, which is looked at first, tells nothing; one of the weights twice does.)"""
    rng = random.Random(states8)
    seen = {True: 0, False: 0}
    for _ in range(400):
        count = rng.choice([1, 2, 5, 40])
        room = 1 << rng.choice([14, 18, 22, 26, 32])
        n = [rng.choice([0, 1, 3, 127, 129, 1000]) for _ in range(count)]
        n[0] = max(n[0], 1)
        p_dtype, g_dtype = ([rng.randrange(2) for _ in range(count)] for _ in range(2))
        place = lambda: A + rng.randrange(room) // 8 * 8      # noqa: E731
        ranges = []

        def ptr(bytes_, written, there=True):
            at = place()
            if there and bytes_:
                ranges.append((at, at + bytes_, written))
            return at
        size = lambda d: 2 if d else 4       # noqa: E731
        k = dict(count=count, n=n, p_dtype=p_dtype, g_dtype=g_dtype)
        k["p"] = [ptr(x * size(d), True) for x, d in zip(n, p_dtype)]
        k["g"] = [ptr(x * size(d), False) for x, d in zip(n, g_dtype)]
        k["m"], k["v"] = ([ptr(x * (1 if states8 else 4), True) for x in n] for _ in range(2))
        if states8:
            k.update(state_kind=1)
            k["m_scale"], k["v_scale"] = ([ptr((x + 127) // 128 * 4, True) for x in n] for _ in range(2))
        k["q"], k["q_scale"] = [ptr(x, True) if rng.random() < 0.7 else None for x in n], ptr(4 * count, False)
        k["lr"], k["step"], k["norm"] = ptr(4, False), ptr(8, False), ptr(4, False)
        wrong = any(a[0] < b[1] and b[0] < a[1] and (a[2] or b[2]) for i, a in enumerate(ranges) for b in ranges[:i])
        seen[wrong] += 1
        if wrong:
            assert adamw(**k) == BAD and "overlap" in fp8.fp8_last_error(), (k, fp8.fp8_last_error())
        else:
            # the first weight once more, behind the others
            twice = {name: list(x) + [x[0] if name in ("p", "n", "p_dtype") else None if name == "q" else A + room + 65536 + 16384 * i] if isinstance(x, list) else x for i, (name, x) in enumerate(k.items())}
            twice.update(count=count + 1, g_dtype=g_dtype + [0], q_scale=A + room + (1 << 20))
            assert adamw(**twice) == BAD, twice
            assert any("two of the weights, p[%d] and p[%d]" % x in fp8.fp8_last_error() for x in ((0, count), (count, 0))), (twice, fp8.fp8_last_error())
    assert min(seen.values()) > 50, seen
