"""Training steps, and decoding, of a transformer's feed-forward block with FP8 products (arXiv 2209.05433, Sections 2 and 4):
E4M3 weights and activations, E5M2 gradients, per-tensor factors, 32-bit master weights.

    python examples/ffn_step.py --block gated --tokens 4096 --width 2048 --inner 6144 --steps 10
    python examples/ffn_step.py --block mlp --tokens 1          # one token, forward only

gated  y = x + (silu(x Wg^T) * (x Wu^T)) Wd^T     fp8_gemm_gated, fp8_gemm_act (residual); backward: fp8_gemm_gated_grad
mlp    y = x + gelu(x W1^T + b1) W2^T + b2        fp8_gemm_act twice; backward: fp8_gemm_act_grad with the bias gradient
both   the input's gradient joins the residual's in fp8_gemm_act, the weights' by fp8_gemm_splitk, and
       fp8_grad_norm / fp8_grad_clip before the update

Tensors that a product writes in FP8 take their factor from the maxima of past steps (delayed scaling); the others are
cast with their own.  Synthetic data: the target is the output of another block of the same kind."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2209_05433_amd as fp8  # noqa: E402

E4M3, E5M2, BF16, F32 = fp8.FP8_E4M3, fp8.FP8_E5M2, fp8.FP8_OUT_BF16, fp8.FP8_OUT_F32


class Cast:
    """FP8 bytes of a tensor and their factor, from the tensor's own maximum; buffers are kept from call to call."""

    def __init__(self, shape, fmt):
        self.fmt = fmt
        self.q = torch.empty(shape, dtype=torch.uint8, device="cuda")
        self.amax, self.scale = torch.zeros(1, device="cuda"), torch.ones(1, device="cuda")
        self.workspace = torch.zeros(fp8.FP8_AMAX_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")

    def __call__(self, x):
        fp8.fp8_amax_scale(x, self.fmt, self.amax, self.scale, self.workspace)
        fp8.fp8_quantize_dscale(x, self.fmt, self.scale, self.q)
        return self


class Delayed:
    """FP8 bytes that a product writes, with a factor from the maxima of the last steps.  The first step has none: its product runs twice,
    the second time with the factor of what the first time saw."""

    def __init__(self, shape, fmt, steps=8):
        self.fmt, self.kind = fmt, fp8.FP8_OUT_E4M3 if fmt == E4M3 else fp8.FP8_OUT_E5M2
        self.q = torch.empty(shape, dtype=torch.uint8, device="cuda")
        self.history, self.scale, self.amax = torch.zeros(steps, device="cuda"), torch.ones(1, device="cuda"), torch.zeros(1, device="cuda")
        self.seen = 0

    def fill(self, product):
        for _ in range(2 if self.seen == 0 else 1):
            fp8.fp8_scale_from_amax_history(self.history, self.fmt, self.scale)
            product(self.q, self.kind, self.scale, self.amax)
            self.history[self.seen % self.history.numel()].copy_(self.amax[0])
        self.seen += 1
        return self


class Block:
    def __init__(self, kind, tokens, width, inner, seed=0):
        self.kind, self.tokens, self.width, self.inner = kind, tokens, width, inner
        gen = torch.Generator(device="cuda").manual_seed(seed)
        first = 2 * inner if kind == "gated" else inner                          # [gate | up], or the up projection
        draw = lambda rows, cols: torch.randn(rows, cols, generator=gen, device="cuda") * cols ** -0.5
        self.W1, self.W2 = draw(first, width), draw(width, inner)
        self.b1, self.b2 = torch.zeros(inner, device="cuda"), torch.zeros(width, device="cuda")
        self.qW1, self.qW2 = Cast(self.W1.shape, E4M3), Cast(self.W2.shape, E4M3)
        self.qx, self.qdy = Cast((tokens, width), E4M3), Cast((tokens, width), E5M2)
        self.h, self.dh = Delayed((tokens, inner), E4M3), Delayed((tokens, first), E5M2)
        self.kept = torch.empty(tokens, first, dtype=torch.bfloat16, device="cuda")          # z, or [g | u], for the backward pass
        self.y = torch.empty(tokens, width, dtype=torch.bfloat16, device="cuda")
        self.dx = torch.empty(tokens, width, dtype=torch.bfloat16, device="cuda")
        self.dW1, self.dW2, self.db1 = torch.empty_like(self.W1), torch.empty_like(self.W2), torch.empty_like(self.b1)
        self.sums = torch.empty(fp8.fp8_gemm_act_grad_workspace_size(tokens, inner), dtype=torch.uint8, device="cuda")
        need = max(fp8.fp8_gemm_splitk_workspace_size(r, c, tokens, True, False) for r, c in (self.W1.shape, self.W2.shape))
        self.slices = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        self.norm, self.norm_workspace = torch.zeros(1, device="cuda"), torch.zeros(fp8.FP8_GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")

    def forward(self, x, train=True):
        """y [tokens, width] for x, both bf16."""
        self.qx(x), self.qW1(self.W1), self.qW2(self.W2)
        kept = self.kept if train else None

        def first(q, kind, scale, amax):
            if self.kind == "gated":
                fp8.fp8_gemm_gated(self.qx.q, E4M3, False, self.qW1.q, E4M3, True, q, kind, self.qx.scale, self.qW1.scale, fp8.FP8_ACT_SILU, kept, scale, amax)
            else:
                fp8.fp8_gemm_act(self.qx.q, E4M3, False, self.qW1.q, E4M3, True, q, kind, self.qx.scale, self.qW1.scale, fp8.FP8_ACT_GELU, self.b1, None, kept, scale, amax)
        self.h.fill(first)
        fp8.fp8_gemm_act(self.h.q, E4M3, False, self.qW2.q, E4M3, True, self.y, BF16, self.h.scale, self.qW2.scale, fp8.FP8_ACT_NONE,
                         None if self.kind == "gated" else self.b2, x)
        return self.y

    def backward(self, dy):
        """Gradients of the weights, biases and (returned) the input, for the gradient dy of the output (bf16)."""
        self.qdy(dy)

        def inner(q, kind, scale, amax):
            operands = (self.qdy.q, E5M2, False, self.qW2.q, E4M3, False, q, kind, self.qdy.scale, self.qW2.scale)
            if self.kind == "gated":
                fp8.fp8_gemm_gated_grad(*operands, fp8.FP8_ACT_SILU, self.kept, scale, amax)
            else:
                fp8.fp8_gemm_act_grad(*operands, fp8.FP8_ACT_GELU, self.kept, self.db1, self.sums, scale, amax)
        self.dh.fill(inner)
        # input: through the first weight, plus what the residual passes on
        fp8.fp8_gemm_act(self.dh.q, E5M2, False, self.qW1.q, E4M3, False, self.dx, BF16, self.dh.scale, self.qW1.scale, fp8.FP8_ACT_NONE, None, dy)
        # weights: sums over the tokens
        fp8.fp8_gemm_splitk(self.dh.q, E5M2, True, self.qx.q, E4M3, False, self.dW1, self.dh.scale, self.qx.scale, self.slices)
        fp8.fp8_gemm_splitk(self.qdy.q, E5M2, True, self.h.q, E4M3, False, self.dW2, self.qdy.scale, self.h.scale, self.slices)
        return self.dx

    def parameters(self, dy):
        """[(parameter, gradient)]; the second bias's gradient is the sum of dy over the tokens."""
        pairs = [(self.W1, self.dW1), (self.W2, self.dW2)]
        return pairs if self.kind == "gated" else pairs + [(self.b1, self.db1), (self.b2, dy.float().sum(0))]

    def update(self, dy, lr, max_norm):
        """One step of clipped gradient descent; the norm before clipping."""
        pairs = self.parameters(dy)
        grads = [g for _, g in pairs]
        fp8.fp8_grad_norm(grads, self.norm, self.norm_workspace)
        fp8.fp8_grad_clip(grads, self.norm, max_norm)
        for p, g in pairs:
            p.sub_(g, alpha=lr)
        return self.norm


def train(kind, tokens, width, inner, steps, lr=0.5, max_norm=1.0):
    """Yields (loss, gradient norm) of each step."""
    x = torch.randn(tokens, width, generator=torch.Generator(device="cuda").manual_seed(7), device="cuda").to(torch.bfloat16)
    target = Block(kind, tokens, width, inner, seed=1).forward(x).float()
    block = Block(kind, tokens, width, inner, seed=2)
    for _ in range(steps):
        error = block.forward(x).float() - target
        dy = (error / tokens).to(torch.bfloat16)                     # of the loss below
        block.backward(dy)
        loss = 0.5 * float(error.square().sum()) / tokens
        yield loss, float(block.update(dy, lr, max_norm))


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--block", choices=("gated", "mlp"), default="gated")
    p.add_argument("--tokens", type=int, default=4096)
    p.add_argument("--width", type=int, default=2048)
    p.add_argument("--inner", type=int, default=6144)
    p.add_argument("--steps", type=int, default=10)
    a = p.parse_args()
    if a.tokens == 1:
        block, x = Block(a.block, 1, a.width, a.inner), torch.randn(1, a.width, device="cuda").to(torch.bfloat16)
        for i in range(a.steps):
            x = block.forward(x, train=False).clone()
            x = (x.float() / x.float().square().mean().sqrt()).to(torch.bfloat16)
            print("token %d  first outputs %s" % (i, ["%.3f" % v for v in x[0, :4].tolist()]))
        return
    for i, (loss, norm) in enumerate(train(a.block, a.tokens, a.width, a.inner, a.steps)):
        print("step %d  loss %.4f  gradient norm %.4f" % (i, loss, norm))


if __name__ == "__main__":
    main()
