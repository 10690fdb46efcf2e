"""The two ends of a training step as a program uses them together: examples/lm_head_step.py against the formulas in 64 bits."""
import importlib.util
import os

import pytest
import torch

import paper_2209_05433_amd as fp8

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
E4M3 = torch.float8_e4m3fn


def example():
    spec = importlib.util.spec_from_file_location("lm_head_step", os.path.join(ROOT, "examples", "lm_head_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("piece", [5000, 1000, 333])
@pytest.mark.parametrize("tokens,width,vocabulary", [(300, 256, 2001), (77, 100, 999)])
def test_losses_and_gradients(tokens, width, vocabulary, piece):
    """Against autograd in 64 bits of the loss of the operands as they are in FP8.  The logits' gradient is rounded to E5M2 once: half a step, 2^-3 of each value
    (2^-17 / y_scale where it is subnormal); so a sum over the vocabulary or the tokens is off by at most 2^-3 times the sum of the terms' magnitudes, and by 2^-19 of
    them for all 32-bit sums and exponentials; the weight's gradient is stored in bf16, 2^-8 of it."""
    ex = example()
    head = ex.Head(tokens, width, vocabulary, piece, seed=3)
    inputs, labels = ex.batch(tokens, vocabulary, torch.Generator(device="cuda").manual_seed(4))
    loss = head.forward(inputs, labels).clone()
    dx = head.backward(inputs, labels)
    x = (head.qx.view(E4M3).double() / float(head.x_scale)).requires_grad_(True)
    w = (head.qW.view(E4M3).double() / float(head.qW_scale[1])).requires_grad_(True)
    z = x @ w.t()
    lse = torch.logsumexp(z, 1)
    each = lse + head.z_weight * lse * lse - z.gather(1, labels.clamp(min=0)[:, None])[:, 0]
    each = torch.where(labels < 0, torch.zeros_like(each), each)
    assert bool(((loss.double() - each).abs() <= 2.0 ** -16 * (1 + each.abs())).all())
    total = each.sum() / (labels >= 0).sum()
    gz, gx, gw = torch.autograd.grad(total, (z, x, w))
    tiny = 2.0 ** -17 / float(head.y_scale)
    size = gz.abs() * (2.0 ** -3 + 2.0 ** -14) + tiny            # (2^-14 for the exponentials of logits and lse of up to 40 and their products)
    assert bool(((dx.double() - gx).abs() <= size @ w.detach().abs() + 2.0 ** -19 * (gz.abs() @ w.detach().abs())).all())
    bound = size.t().contiguous() @ x.detach().abs() * (1 + 2.0 ** -7)
    assert bool(((head.grads[1].double() - gw).abs() <= bound + 2.0 ** -8 * gw.abs() + 1e-30).all())
    want = torch.zeros(vocabulary, width, dtype=torch.float64, device="cuda").index_add_(0, inputs, dx.double())
    assert bool(((head.grads[0].double() - want).abs() <= 2.0 ** -20 * want.abs() + 1e-9).all())


@pytest.mark.parametrize("states", ["fp8", "f32"])
def test_an_update(states):
    """The weights after a step against the formulas, and their FP8 copies and maxima against the weights."""
    ex = example()
    head = ex.Head(200, 128, 1501, 600, states, seed=5)
    inputs, labels = ex.batch(200, 1501, torch.Generator(device="cuda").manual_seed(6))
    head.forward(inputs, labels)
    head.backward(inputs, labels)
    before, grads = [p.double() for p in head.params], [g.double() for g in head.grads]
    scale = head.qW_scale.clone()
    norm = float(head.update(1e-2, 0.5))
    assert abs(norm - float(torch.sqrt(sum(g.square().sum() for g in grads)))) <= 2.0 ** -22 * norm
    c = min(1.0, 0.5 / (norm + 1e-6))
    for p, old, g, decay in zip(head.params, before, grads, (0.0, 0.01)):
        # the first step from states of 0: m / (1 - b1) is the gradient, sqrt(v / (1 - b2)) its magnitude
        u = g * c / ((g * c).abs() + 1e-8)
        want = old - float(head.lr) * (u + decay * old)
        assert bool(((p.double() - want).abs() <= 2.0 ** -24 * want.abs() + 1e-2 * 2.0 ** -18).all())
    w = head.params[1]
    assert float(head.qW_amax[1]) == float(w.abs().max()) and float(head.qW_amax[0]) == 0.0
    assert torch.equal(head.qW.view(E4M3).float(), (w * scale[1]).clamp(-448, 448).to(E4M3).float())


@pytest.mark.parametrize("states", ["fp8", "f32"])
def test_training_steps_run(states):
    runs = list(example().train(512, 128, 1000, 6, 400, states))
    assert len(runs) == 6 and all(l == l and abs(l) < 100 and n == n and n > 0 for l, n in runs)


def test_a_step_in_a_graph():
    """Everything between the choice of the batch and the next one's, captured and replayed, against the same steps taken eagerly."""
    ex = example()
    a, b = (ex.Head(256, 128, 1500, 700, seed=7) for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(8)
    batches = [ex.batch(256, 1500, gen) for _ in range(4)]
    inputs, labels = (t.clone() for t in batches[0])

    def kernels(h, i, y):
        """(the embedding's gradient, whose additions have no fixed order, left out)"""
        h.forward(i, y)
        h.dloss.fill_(1.0 / 256)
        h.y_scale.fill_(28672.0 * 256)
        for k, (lo, hi) in enumerate(h.pieces):
            d, w = h.y[:256 * (hi - lo)].view(256, hi - lo), h.qW[lo:hi]
            fp8.fp8_gemm_xent_grad(h.qx, 0, False, w, 0, True, d, fp8.FP8_OUT_E5M2, h.x_scale, h.qW_scale[1:], y, h.lse, h.dloss, first=lo, z_weight=h.z_weight, sD=h.y_scale)
            fp8.fp8_gemm_act(d, 1, False, w, 0, False, h.dx, 0, h.y_scale, h.qW_scale[1:], 0, None, h.dx if k else None)
            fp8.fp8_gemm_ex(d, 1, True, h.qx, 0, False, h.grads[1][lo:hi], h.y_scale, h.x_scale)
        h.update(1e-2)
    warm = ex.Head(256, 128, 1500, 700, seed=7)
    kernels(warm, inputs, labels)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kernels(a, inputs, labels)
    for i, y in batches:
        inputs.copy_(i), labels.copy_(y)
        kernels(b, i, y)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in ("loss", "lse", "dx", "qW", "qW_amax", "norm", "step"):
            assert torch.equal(getattr(a, name), getattr(b, name)), name
        for xs, ys in ((a.params, b.params), (a.m, b.m), (a.v, b.v), (a.grads, b.grads)):
            assert all(torch.equal(p, q) for p, q in zip(xs, ys))
