"""A stack of residual blocks trained, and served with adapters, with the layer operators of gemm2m.

    python examples/fp8_block_training.py

One block:  H = X + (what the block before it computed),  N = norm(H),  F = relu(N Wu^T),  next block's summand F Wd^T.
    training   the norm writes its 8-bit forms itself (no 16-bit N); its backward pass joins the gradient of the residual path;
               all gradients are clipped by their common norm before the orthogonalised updates
    serving    tokens of many requests at once, each with its request's low-rank update of Wu, or none
torch does what is elementwise; the norms, the products, the clipping, the adapters and the orthogonalisation are the library's.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from examples.fp8_layer_training import Fp8Linear  # noqa: E402
from paper_2609_05419_b200 import binding as g2m  # noqa: E402

EPS = 1e-6


class Norm:
    """Root-mean-square norm whose output is the operand of 8-bit products."""

    def __init__(self, width):
        self.w = torch.ones(width, device="cuda")
        self.dw = torch.zeros_like(self.w)

    def forward(self, x, summand):
        """The stream x + summand, and the 8-bit forms of its norm along the rows and along the columns."""
        tokens, width = x.shape
        self.h, self.rstd = torch.empty_like(x), torch.empty(tokens, device="cuda")
        rows, columns = g2m.fp8_empty(tokens, width), g2m.fp8_empty(width, tokens)
        g2m.rms_norm(x, self.w, R=summand, H=self.h, Q=rows[0], S=rows[1], Qt=columns[0], St=columns[1], rstd=self.rstd, eps=EPS)
        return self.h, rows, columns

    def backward(self, dn, dh):
        """The stream's gradient in front of the norm, from the norm's (dn) and the one that came along the residual path (dh)."""
        dx = torch.empty_like(dn)
        g2m.rms_norm_backward(dn, self.h, self.w, self.rstd, dx, dR=dh, dW=self.dw, add=True)
        return dx


class Block:
    def __init__(self, width, inner, generator):
        self.norm = Norm(width)
        self.up, self.down = Fp8Linear(width, inner, generator), Fp8Linear(inner, width, generator)

    def forward(self, x, summand):
        h, rows, (self.up.qxt, self.up.sxt) = self.norm.forward(x, summand)
        f = torch.empty(x.shape[0], self.up.w.shape[0], dtype=torch.bfloat16, device="cuda")
        g2m.fp8_gemm(*rows, self.up.qw, self.up.sw, f)
        self.active = f > 0
        return h, self.down.forward(torch.relu(f))

    def backward(self, dh):
        """dh: gradient of the stream behind the block, that is of H and of the block's summand alike."""
        df = self.down.backward(dh)
        return self.norm.backward(self.up.backward(torch.where(self.active, df, torch.zeros_like(df))), dh)

    def serve(self, x, summand, adapters, index):
        """The same without what only a backward pass needs, plus scale (N A^T) B^T of each token's adapter on the way to F."""
        n, h = torch.empty_like(x), torch.empty_like(x)
        q, s = g2m.fp8_empty(*x.shape)
        g2m.rms_norm(x, self.norm.w, R=summand, H=h, Y=n, Q=q, S=s, eps=EPS)
        f = torch.empty(x.shape[0], self.up.w.shape[0], dtype=torch.bfloat16, device="cuda")
        g2m.fp8_gemm(q, s, self.up.qw, self.up.sw, f)
        a, b, scales = adapters
        g2m.adapter_add(n, a, b, index, f, C=f, scales=scales)
        return h, self.down.forward(torch.relu(f))


class Stack:
    def __init__(self, blocks, width, inner, generator):
        self.blocks = [Block(width, inner, generator) for _ in range(blocks)]

    def gradients(self):
        return [t for b in self.blocks for t in (b.up.dw, b.down.dw, b.norm.dw)]

    def forward(self, x):
        summand = torch.zeros_like(x)
        for block in self.blocks:
            x, summand = block.forward(x, summand)
        return x, summand

    def backward(self, dh):
        for block in reversed(self.blocks):
            dh = block.backward(dh)
        return dh

    def serve(self, x, adapters, index):
        summand = torch.zeros_like(x)
        for block, mine in zip(self.blocks, adapters):
            x, summand = block.serve(x, summand, mine, index)
        return x + summand

    def step(self, rate, limit, norm):
        g2m.clip_gradients(self.gradients(), limit, norm=norm)
        for block in self.blocks:
            block.up.step(rate)
            block.down.step(rate)
            block.norm.w.add_(block.norm.dw, alpha=-rate)
            block.norm.dw.zero_()

    def workspace(self, tokens, rank, many):
        """One workspace that is large enough for every call."""
        sizes = [(g2m.OP_FP8_GEMM, 1, 1, 1), (g2m.OP_CLIP_GRADIENTS, len(self.gradients()), 1, 1), (g2m.OP_ADAPTER_ADD, tokens, rank, many)]
        for block in self.blocks:
            width = block.norm.w.numel()
            sizes += [(g2m.OP_RMS_NORM, tokens, width, 1), (g2m.OP_RMS_NORM_BACKWARD, tokens, width, 1)]
            sizes += [(g2m.OP_NEWTON_SCHULZ, *layer.w.shape, 1) for layer in (block.up, block.down)]
        return torch.zeros(max(g2m.workspace_bytes(*size, 1) for size in sizes), dtype=torch.uint8, device="cuda")


def make_adapters(blocks, many, rank, width, inner, generator):
    """For every block (A, B, scales) of `many` adapters."""
    randn = lambda *shape: torch.randn(*shape, generator=generator, device="cuda")
    return [((randn(many, rank, width) * width ** -0.5).bfloat16(), (randn(many, inner, rank) * 0.1).bfloat16(), torch.full((many,), 2.0, device="cuda"))
            for _ in range(blocks)]


def train(steps=20, tokens=400, width=264, inner=520, blocks=2, rate=0.03, limit=1.0, seed=0):
    """Fits random targets of random inputs; returns the loss and the norm of the gradients of every step, and what serving gives afterwards."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    stack = Stack(blocks, width, inner, gen)
    adapters = make_adapters(blocks, 5, 8, width, inner, gen)
    workspace = stack.workspace(tokens, 8, 5)
    g2m.set_workspace(workspace)
    x = torch.randn(tokens, width, generator=gen, device="cuda").bfloat16()
    target = torch.randn(tokens, width, generator=gen, device="cuda")
    losses, norms = [], []
    try:
        for _ in range(steps):
            h, summand = stack.forward(x)
            error = h.float() + summand.float() - target
            losses.append((error * error).mean())
            stack.backward((error * (2.0 / error.numel())).bfloat16())
            norms.append(torch.empty((), device="cuda"))
            stack.step(rate, limit, norms[-1])
        index = torch.randint(-1, 5, (tokens,), generator=gen, device="cuda").to(torch.int32)
        served = stack.serve(x, adapters, index)
        g2m.device_status()
        return [float(v) for v in losses], [float(v) for v in norms], served
    finally:
        torch.cuda.synchronize()
        g2m.set_workspace(None)


if __name__ == "__main__":
    losses, norms, _ = train(40)
    for i in range(0, 40, 5):
        print(f"step {i:3d}  loss {losses[i]:.4f}  norm of the gradients {norms[i]:.4f}")
