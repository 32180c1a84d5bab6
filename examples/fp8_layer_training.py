"""A two-layer network trained with the layer operators of gemm2m: every product in 8-bit floating point with block scales, every
weight update orthogonalised by Newton-Schulz steps.

    python examples/fp8_layer_training.py

One step of a layer Y = X W^T (X: tokens x in, W: out x in):
    forward          X  -> 8 bits, 1 x 128 blocks;  W -> 8 bits, 128 x 128 blocks, both orientations;   Y = X W^T
    backward         dY -> 8 bits, both orientations;  dX = dY W (the transposed weights);  dW += dY^T X (32 bits)
    update           M <- beta M + dW;  W <- W - rate sqrt(max(1, out / in)) orthogonalise(M)
torch does what is elementwise; the products, the quantisation and the orthogonalisation are the library's.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_05419_b200 import binding as g2m  # noqa: E402


class Fp8Linear:
    """A linear layer without bias: 32-bit weights, 8-bit products."""

    def __init__(self, n_in, n_out, generator):
        self.w = torch.randn(n_out, n_in, generator=generator, device="cuda") * n_in ** -0.5
        self.dw = torch.zeros_like(self.w)
        self.momentum = torch.zeros_like(self.w)
        self.update = torch.empty(n_out, n_in, dtype=torch.bfloat16, device="cuda")
        self.qw, self.sw = g2m.fp8_empty(n_out, n_in, block_rows=128)
        self.qwt, self.swt = g2m.fp8_empty(n_in, n_out, block_rows=128)
        self.quantise_weights()

    def quantise_weights(self):
        g2m.fp8_quantise(self.w, self.qw, self.sw, self.qwt, self.swt, block_rows=128)

    def forward(self, x):
        tokens, n_in = x.shape
        qx, sx = g2m.fp8_empty(tokens, n_in)
        self.qxt, self.sxt = g2m.fp8_empty(n_in, tokens)           # kept for the weight gradient, instead of x
        g2m.fp8_quantise(x, qx, sx, self.qxt, self.sxt)
        y = torch.empty(tokens, self.w.shape[0], dtype=torch.bfloat16, device="cuda")
        g2m.fp8_gemm(qx, sx, self.qw, self.sw, y)
        return y

    def backward(self, dy, need_dx=True):
        tokens, n_out = dy.shape
        q, s = g2m.fp8_empty(tokens, n_out)
        qt, st = g2m.fp8_empty(n_out, tokens)
        g2m.fp8_quantise(dy, q, s, qt, st)
        g2m.fp8_gemm(qt, st, self.qxt, self.sxt, self.dw, C=self.dw, b_block=1)      # added to the earlier micro-batches' sum
        if not need_dx:
            return None
        dx = torch.empty(tokens, self.w.shape[1], dtype=torch.bfloat16, device="cuda")
        g2m.fp8_gemm(q, s, self.qwt, self.swt, dx)
        return dx

    def step(self, rate, beta=0.9):
        n_out, n_in = self.w.shape
        self.momentum.mul_(beta).add_(self.dw)
        g2m.newton_schulz(self.momentum, self.update)
        self.w.add_(self.update, alpha=-rate * max(1.0, n_out / n_in) ** 0.5)
        self.dw.zero_()
        self.quantise_weights()


def workspace_for(layers):
    """One workspace that is large enough for every call on these layers."""
    need = g2m.workspace_bytes(g2m.OP_FP8_GEMM, 1, 1, 1, 1)
    for layer in layers:
        need = max(need, g2m.workspace_bytes(g2m.OP_NEWTON_SCHULZ, *layer.w.shape, 1, 1))
    return torch.zeros(need, dtype=torch.uint8, device="cuda")


def train(steps=30, tokens=512, n_in=384, hidden=520, n_out=256, rate=0.05, micro_batches=2, seed=0):
    """Fits a random teacher network; returns the loss of every step."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    teacher = [torch.randn(hidden, n_in, generator=gen, device="cuda") * n_in ** -0.5,
               torch.randn(n_out, hidden, generator=gen, device="cuda") * hidden ** -0.5]
    layers = [Fp8Linear(n_in, hidden, gen), Fp8Linear(hidden, n_out, gen)]
    workspace = workspace_for(layers)
    g2m.set_workspace(workspace)
    losses = []
    try:
        for _ in range(steps):
            total = 0.0
            for _ in range(micro_batches):
                x = torch.randn(tokens, n_in, generator=gen, device="cuda")
                target = torch.relu(x @ teacher[0].t()) @ teacher[1].t()
                h = layers[0].forward(x.bfloat16())
                y = layers[1].forward(torch.relu(h))
                error = y.float() - target
                total = total + (error * error).mean() / micro_batches
                dy = error * (2.0 / (error.numel() * micro_batches))
                dh = layers[1].backward(dy)
                layers[0].backward(torch.where(h > 0, dh, torch.zeros_like(dh)), need_dx=False)
            for layer in layers:
                layer.step(rate)
            losses.append(total)
        g2m.device_status()
        return [float(v) for v in losses]
    finally:
        torch.cuda.synchronize()
        g2m.set_workspace(None)


if __name__ == "__main__":
    for i, loss in enumerate(train(60)):
        if i % 5 == 0 or i == 59:
            print(f"step {i:3d}  loss {loss:.4f}")
