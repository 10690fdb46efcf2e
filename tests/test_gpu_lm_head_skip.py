"""examples/lm_head_step.py where a step is skipped because its gradients' norm is not finite: everything stays as it was, the weights' FP8 bytes with the factor they were made by."""
import math

import pytest
import torch

from test_gpu_lm_head_example import E4M3, example

pytestmark = pytest.mark.gpu


def state_of(head):
    return [x.clone() for x in [*head.params, *head.m, *head.v, *head.scales[0], *head.scales[1], head.qW, head.qW_scale, head.qW_amax, head.step]]


def steps(head, ex, gen, count):
    for _ in range(count):
        inputs, labels = ex.batch(head.tokens, head.vocabulary, gen)
        head.forward(inputs, labels)
        head.backward(inputs, labels)
        head.update(1e-2)


def consistent(head):
    """(saturating, to the nearest: one rounding, as the weights are in 32 bits)"""
    return torch.equal(head.qW.view(E4M3).float(), (head.params[1] * head.qW_scale[1]).clamp(-448, 448).to(E4M3).float())


@pytest.mark.parametrize("states", ["fp8", "f32"])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("before", [0, 2])
def test_a_skipped_step(states, bad, before):
    ex = example()
    head, gen = ex.Head(200, 128, 1501, 600, states, seed=5), torch.Generator(device="cuda").manual_seed(6)
    steps(head, ex, gen, before)
    assert int(head.step) == before and consistent(head)
    kept = state_of(head)
    for where in (0, 1, 1):
        head.grads[where].view(-1)[1234] = bad
        head.update(1e-2)
        assert all(torch.equal(a, b) for a, b in zip(kept, state_of(head)))
        assert int(head.step) == before and consistent(head)
        # (the bad element goes with the next backward pass)
    steps(head, ex, gen, 2)
    assert int(head.step) == before + 2 and consistent(head) and all(bool(torch.isfinite(p).all()) for p in head.params)


def test_skipped_steps_in_a_graph():
    """The same update captured, with finite and infinite gradients between the replays, against eager ones."""
    ex = example()
    a, b = (ex.Head(100, 64, 501, 300, seed=7) for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(8)
    grads = [[torch.randn(g.shape, generator=gen, device="cuda").to(g.dtype) for g in a.grads] for _ in range(5)]
    grads[0][1][3, 3] = grads[2][0][5, 5] = math.inf
    grads[3][1][0, 0] = math.nan
    warm = ex.Head(100, 64, 501, 300, seed=7)
    warm.update(1e-2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.update(1e-2)
    counts = []
    for new in grads:
        for head in (a, b):
            for g, x in zip(head.grads, new):
                g.copy_(x)
        b.update(1e-2)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(state_of(a), state_of(b))) and consistent(a)
        counts.append(int(a.step))
    assert counts == [0, 1, 1, 1, 2]
