"""One workspace, sized for the largest call and not a byte more, serves smaller calls of the same operator: on the GPU, with a guard behind it."""
import pytest
import torch

from paper_2609_05419_b200 import binding as b

pytestmark = pytest.mark.gpu

from test_gpu_adapters import operands, plain, room  # noqa: E402


class Guarded:
    """A workspace at the start of a larger store, which has to stay as it was behind it."""

    def __init__(self, size):
        self.size, self.store = size, torch.full((size + (1 << 16),), 0xa5, dtype=torch.uint8, device="cuda")
        self.store[:min(size, 4096)] = 0

    def __enter__(self):
        b.set_workspace(self.store[:self.size])

    def __exit__(self, *exc):
        torch.cuda.synchronize()
        b.set_workspace(None)
        assert exc[0] is not None or bool((self.store[self.size:] == 0xa5).all())


def test_adapters_of_a_decoding_batch_in_the_workspace_of_the_prompts():
    k, n, many, rank = 96, 136, 8, 16
    with Guarded(b.workspace_bytes(b.OP_ADAPTER_ADD, 1024, rank, many, 1)):
        for tokens, used, smaller in ((1024, 8, 16), (256, 8, 16), (256, 1, 16), (128, 8, 16), (207, 1, 7), (1, 1, 1), (300, 2, 16), (257, 8, 3)):
            x, a, w, index, c, scales, _ = operands(tokens, k, n, used, smaller, torch.bfloat16, tokens, ranks=False)
            d = torch.empty_like(c)
            b.adapter_add(x, a, w, index, d, C=c, scales=scales)
            b.device_status()
            want, size, beside = plain(x, a, w, index, c, scales, None)
            assert bool(((d.double() - want).abs() <= room(k, smaller, want, size, beside, torch.bfloat16, torch.bfloat16)).all())


@pytest.mark.parametrize("tokens,many,rank", [(1, 1, 1), (16, 1, 16), (207, 1, 128), (255, 1, 33), (256, 300, 128), (48, 24, 64), (257, 1, 128), (1000, 300, 24)])
def test_adapters_stay_inside_their_own_workspace(tokens, many, rank):
    x, a, w, index, c, scales, _ = operands(tokens, 2048, 40, many, rank, torch.float16, 7, ranks=False)
    with Guarded(b.workspace_bytes(b.OP_ADAPTER_ADD, tokens, rank, many, 1)):
        b.adapter_add(x, a, w, index, torch.empty_like(c), C=c, scales=scales)
        b.device_status()


def test_gradients_of_the_norm_in_the_workspace_of_wider_and_longer_ones():
    with Guarded(b.workspace_bytes(b.OP_RMS_NORM_BACKWARD, 4096, 8193, 1, 1)):
        for rows, cols in ((4096, 8193), (4096, 8192), (4096, 5120), (2500, 512), (300, 5121), (1, 8000)):
            h, dy = torch.randn(rows, cols, device="cuda").bfloat16(), torch.randn(rows, cols, device="cuda").bfloat16()
            rstd = torch.rsqrt(h.float().square().mean(1) + 1e-6)
            dw = torch.empty(cols, device="cuda")
            b.rms_norm_backward(dy, h, None, rstd, torch.empty_like(h), dW=dw)
            terms = dy.double() * h.double() * rstd.double()[:, None]
            # fewer than rows + 160 additions of a column in 32 bits
            assert bool(((dw.double() - terms.sum(0)).abs() <= (rows + 160) * 2.0 ** -24 * terms.abs().sum(0)).all())
