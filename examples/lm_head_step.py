"""Training steps of a language model's two ends with FP8 products (arXiv 2209.05433, Sections 2 and 4): the projection onto the vocabulary with
its loss, and the update of the weights.  E4M3 weights and activations, E5M2 gradients, 32-bit master weights.

    python examples/lm_head_step.py --tokens 4096 --width 2048 --vocabulary 50257 --steps 10
    python examples/lm_head_step.py --states f32 --piece 16384

forward    fp8_gemm_xent: the loss of every token out of x and the vocabulary's weight, no logits in memory
backward   a piece of the vocabulary at a time: fp8_gemm_xent_grad (E5M2, its factor from the bound |y| <= dloss), the tokens' gradient added up by
           fp8_gemm_act with the residual in place, the weight's rows by fp8_gemm_ex
update     fp8_grad_norm, then fp8_adamw with the clipping in it; it leaves the weights' FP8 bytes for the next step's products, with factors from
           their last maxima

The trained model is a token's vector times the vocabulary's weight: x = rows of an embedding of its own.  Synthetic data: the next token is a fixed function of
the one before."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2209_05433_amd as fp8  # noqa: E402

E4M3, E5M2, BF16, F32 = fp8.FP8_E4M3, fp8.FP8_E5M2, fp8.FP8_OUT_BF16, fp8.FP8_OUT_F32


class Head:
    """Embedding and vocabulary projection of `vocabulary` tokens, `width` wide; batches of `tokens`, pieces of `piece` columns."""

    def __init__(self, tokens, width, vocabulary, piece=16384, states="fp8", z_weight=1e-4, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device="cuda")       # noqa: E731
        self.tokens, self.width, self.vocabulary, self.z_weight = tokens, width, vocabulary, z_weight
        self.pieces = [(i, min(i + piece, vocabulary)) for i in range(0, vocabulary, piece)]
        self.params = [torch.randn(vocabulary, width, generator=gen, device="cuda"), torch.randn(vocabulary, width, generator=gen, device="cuda") * width ** -0.5]
        self.grads = [new(vocabulary, width), new(vocabulary, width, dtype=torch.bfloat16)]
        # states of zeros, and the weights' copies in FP8 (the embedding is read in 32 bits)
        self.states8 = states == "fp8"
        self.m, self.v = ([new(vocabulary * width, dtype=torch.uint8 if self.states8 else torch.float32) for _ in range(2)] for _ in range(2))
        blocks = (vocabulary * width + fp8.FP8_STATE_BLOCK - 1) // fp8.FP8_STATE_BLOCK
        self.scales = [[torch.ones(blocks, device="cuda") for _ in range(2)] for _ in range(2)]
        self.qW, self.qW_scale, self.qW_amax, self.next_scale = new(vocabulary, width, dtype=torch.uint8), torch.ones(2, device="cuda"), new(2), new(2)
        self.step, self.lr = new(1, dtype=torch.int64), new(1)
        # the tokens' vectors
        self.qx, self.x_amax, self.x_scale = new(tokens, width, dtype=torch.uint8), new(1), torch.ones(1, device="cuda")
        self.workspace = new(fp8.FP8_AMAX_WORKSPACE_BYTES, dtype=torch.uint8)
        fp8.fp8_amax_scale(self.params[1], E4M3, self.qW_amax[1:], self.qW_scale[1:], self.workspace)
        fp8.fp8_quantize_dscale(self.params[1], E4M3, self.qW_scale[1:], self.qW)
        # loss and gradients
        self.loss, self.lse = new(tokens), new(tokens)
        self.loss_workspace = new(fp8.fp8_gemm_xent_workspace_size(tokens, vocabulary), dtype=torch.uint8)
        self.y, self.y_scale, self.dloss = new(tokens * min(piece, vocabulary), dtype=torch.uint8), new(1), new(1)
        self.dx = new(tokens, width)
        self.norm, self.norm_workspace = new(1), new(fp8.FP8_GRAD_NORM_WORKSPACE_BYTES, dtype=torch.uint8)

    def forward(self, inputs, labels):
        """The losses of the tokens (labels < 0: 0), for token numbers and labels of 64 bits."""
        x = self.params[0][inputs]
        fp8.fp8_amax_scale(x, E4M3, self.x_amax, self.x_scale, self.workspace)
        fp8.fp8_quantize_dscale(x, E4M3, self.x_scale, self.qx)
        fp8.fp8_gemm_xent(self.qx, E4M3, False, self.qW, E4M3, True, labels, self.loss, self.lse, self.loss_workspace, self.x_scale, self.qW_scale[1:], z_weight=self.z_weight)
        return self.loss

    def backward(self, inputs, labels):
        """Gradients of the mean loss over the tokens with a label, of both parameters (in self.grads) and of x (returned)."""
        self.dloss.copy_(1.0 / (labels >= 0).sum().clamp(min=1))
        # |y| <= dloss (1 + 2 z_weight lse), which leaves half the range for the last term
        self.y_scale.copy_(28672.0 / self.dloss)
        for i, (lo, hi) in enumerate(self.pieces):
            y, qW = self.y[:self.tokens * (hi - lo)].view(self.tokens, hi - lo), self.qW[lo:hi]
            fp8.fp8_gemm_xent_grad(self.qx, E4M3, False, qW, E4M3, True, y, fp8.FP8_OUT_E5M2, self.x_scale, self.qW_scale[1:], labels, self.lse, self.dloss, first=lo,
                                   z_weight=self.z_weight, sD=self.y_scale)
            fp8.fp8_gemm_act(y, E5M2, False, qW, E4M3, False, self.dx, F32, self.y_scale, self.qW_scale[1:], fp8.FP8_ACT_NONE, None, self.dx if i else None)
            fp8.fp8_gemm_ex(y, E5M2, True, self.qx, E4M3, False, self.grads[1][lo:hi], self.y_scale, self.x_scale)
        self.grads[0].zero_().index_add_(0, inputs, self.dx)
        return self.dx

    def update(self, lr, max_norm=1.0):
        """One step of AdamW; the norm before clipping."""
        self.lr.fill_(lr)
        fp8.fp8_grad_norm(self.grads, self.norm, self.norm_workspace)
        # a norm that is not finite leaves weights, states and FP8 bytes as they are: the count too, and the factor that the bytes were made by (decided on the device, for graphs)
        goes = torch.isfinite(self.norm)
        self.step.add_(goes)
        fp8.fp8_scale_from_amax_n(self.qW_amax, E4M3, self.next_scale)
        self.qW_scale.copy_(torch.where(goes, self.next_scale, self.qW_scale))
        states = dict(m_scale=self.scales[0], v_scale=self.scales[1], seed=17) if self.states8 else {}
        fp8.fp8_adamw(self.params, self.grads, self.m, self.v, self.step, self.lr, 0.9, 0.95, 1e-8, [0.0, 0.01], self.norm, max_norm, q=[None, self.qW], q_scale=self.qW_scale,
                      q_amax=self.qW_amax, flags=fp8.FP8_ADAMW_SKIP_NONFINITE, **states)
        return self.norm


def batch(tokens, vocabulary, gen):
    inputs = torch.randint(0, vocabulary, (tokens,), generator=gen, device="cuda")
    labels = (inputs * 31 + 7) % vocabulary
    return inputs, torch.where(torch.rand(tokens, generator=gen, device="cuda") < 0.05, -100, labels)


def train(tokens, width, vocabulary, steps, piece=16384, states="fp8", lr=1e-2, seed=0):
    """Yields (mean loss, gradient norm) of each step."""
    head, gen = Head(tokens, width, vocabulary, piece, states, seed=seed), torch.Generator(device="cuda").manual_seed(seed + 1)
    for _ in range(steps):
        inputs, labels = batch(tokens, vocabulary, gen)
        loss = float(head.forward(inputs, labels).sum() / (labels >= 0).sum())
        head.backward(inputs, labels)
        yield loss, float(head.update(lr))


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--tokens", type=int, default=4096)
    p.add_argument("--width", type=int, default=2048)
    p.add_argument("--vocabulary", type=int, default=50257)
    p.add_argument("--piece", type=int, default=16384)
    p.add_argument("--states", choices=("fp8", "f32"), default="fp8")
    p.add_argument("--steps", type=int, default=10)
    a = p.parse_args()
    for i, (loss, norm) in enumerate(train(a.tokens, a.width, a.vocabulary, a.steps, a.piece, a.states)):
        print("step %d  loss %.4f  gradient norm %.4f" % (i, loss, norm))


if __name__ == "__main__":
    main()
