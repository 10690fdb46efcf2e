"""AdamW where a workgroup takes several chunks of 4096 elements, which it does beyond 65536 chunks in a launch: small tensors side by side in one workgroup's share, with and without copies,
each with a maximum of its own, before, between and behind two large ones."""
import pytest
import torch

import paper_2209_05433_amd as fp8

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
BLOCK, CHUNK = fp8.FP8_STATE_BLOCK, 4096
SMALL = [4096, 1, 77, 4095, 4096, 300, 8192, 0, 5, 4097, 128, 129, 10001]
LARGE = (500_000_007, 310_000_000)
SIZES = SMALL + [LARGE[0]] + SMALL + [LARGE[1]] + SMALL[::-1]
COUNT = len(SIZES)
assert COUNT <= 50 and 3 * 65536 < sum(-(-n // CHUNK) for n in SIZES) < 4 * 65536
U = 2.0 ** -24


class State:
    def __init__(self, states8, empty=()):
        """(empty: tensors that are there with no elements)"""
        gen = torch.Generator(device="cuda").manual_seed(1)
        self.p, self.g, self.m, self.v, self.ms, self.vs, self.q = ([] for _ in range(7))
        for i, n in enumerate(SIZES):
            p = torch.empty(n, dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.05, generator=gen)
            g = torch.empty(n, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1e-2, generator=gen)
            p.clamp_(-1, 1)
            if n:
                # the largest weight, which nothing moves
                at = n // 2 if n < 1 << 20 else n - 2
                p[at], g[at] = 2.0 + i / 16, 0.0
            keep = (lambda x: x[:0]) if i in empty else (lambda x: x)
            self.p.append(keep(p)), self.g.append(keep(g))
            n = self.p[-1].numel()
            new = lambda count, dtype: torch.zeros(count, dtype=dtype, device="cuda")      # noqa: E731
            self.m.append(new(n, torch.uint8 if states8 else torch.float32)), self.v.append(new(n, torch.uint8 if states8 else torch.float32))
            if states8:
                self.ms.append(new((n + BLOCK - 1) // BLOCK, torch.float32) + 1), self.vs.append(new((n + BLOCK - 1) // BLOCK, torch.float32) + 1)
            self.q.append(new(n, torch.uint8) if i % 4 != 2 else None)
        self.amax = torch.full((COUNT,), 99.0, device="cuda")
        self.scale = 100.0 + torch.arange(COUNT, device="cuda", dtype=torch.float32)
        self.more = dict(m_scale=self.ms, v_scale=self.vs, seed=77) if states8 else {}

    def step(self):
        t, lr = torch.full((1,), 3, dtype=torch.int64, device="cuda"), torch.full((1,), 1e-3, device="cuda")
        fp8.fp8_adamw(self.p, self.g, self.m, self.v, t, lr, 0.9, 0.95, 1e-6, q=self.q, q_scale=self.scale, q_amax=self.amax, **self.more)

    def of(self, i):
        return [x[i] for x in (self.p, self.m, self.v, *((self.ms, self.vs) if self.ms else ()), self.q) if x[i] is not None]


@pytest.mark.parametrize("states8", [False, True])
def test_several_chunks_a_workgroup(states8):
    large = [i for i, n in enumerate(SIZES) if n in LARGE]
    x = State(states8)
    old = [p[:1 << 20].clone() if i in large else p.clone() for i, p in enumerate(x.p)]
    tails = {i: x.p[i][-(1 << 20):].clone() for i in large}
    x.step()
    # every tensor's maximum is its own, nothing of its neighbours' in the workgroup's share
    want = [0.0 if SIZES[i] == 0 or x.q[i] is None else 2.0 + i / 16 for i in range(COUNT)]
    assert x.amax.tolist() == want, [(i, a, b) for i, (a, b) in enumerate(zip(x.amax.tolist(), want)) if a != b]
    # the small ones as in a launch of few chunks
    y = State(states8, empty=large)
    y.step()
    for i in range(COUNT):
        if i not in large:
            assert all(torch.equal(a, b) for a, b in zip(x.of(i), y.of(i))), i
            assert x.q[i] is None or float(x.amax[i]) == float(y.amax[i])
    del y
    # the large ones' beginnings and ends against the formula: from states of 0, m' / (1 - b1^3) = 0.1 g / 0.271, v' = 0.05 g^2; 32u of the update, half an ulp of a bf16 weight
    for i in large:
        for new, before, g in ((x.p[i][:1 << 20], old[i], x.g[i][:1 << 20]), (x.p[i][-(1 << 20):], tails[i], x.g[i][-(1 << 20):])):
            g, before = g.double(), before.double()
            u = 1e-3 * (0.1 * g / (1 - 0.9 ** 3)) / ((0.05 * g * g / (1 - 0.95 ** 3)).sqrt() + 1e-6)
            assert bool(((new.double() - (before - u)).abs() <= 2.0 ** -8 * (before - u).abs() + 64 * U * u.abs() + 1e-30).all())
            assert float((new.double() - before).abs().max()) > 0
        # copies: of the weights before they are rounded to 16 bits, so off by that and by half a step of E4M3
        if x.q[i] is not None:
            for part in (slice(0, 1 << 20), slice(SIZES[i] - (1 << 20), SIZES[i])):
                want_q = (x.p[i][part].double() * float(x.scale[i])).clamp(-448, 448)
                got = x.q[i][part].view(F8).double()
                assert bool(((got - want_q).abs() <= want_q.abs() * (2.0 ** -4 + 2.0 ** -7) + 2.0 ** -10).all())
        assert all(bool((s[-1000:] != 1).all()) for s in ((x.ms[i][:-1], x.vs[i][:-1]) if states8 else ()))
