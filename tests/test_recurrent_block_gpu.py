"""The example that runs the recurrence, the gated feed-forward product and the
4-bit products together: training lowers the loss, its gradients are those of
the same block written in torch (fp32, autograd), and serving token by token
gives what the whole sequence gives."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def example():
    import torch
    from paper_1810_09958_gb300 import build
    build.build()
    torch.cuda.set_device(0)
    import recurrent_block
    return recurrent_block


def test_training_lowers_the_loss(example):
    _, losses = example.train(D=256, H=192, F=320, T=40, B=3, steps=12)
    assert losses[-1] < 0.5 * losses[0], losses


def test_gradients_are_autograds(example):
    """Every intermediate of the block is rounded to bf16 (2^-8 of itself), about
    six of them between a weight and the output; their errors add up
    independently, to about 2^-8 sqrt(6) = 1% of the gradient's norm; 3% is
    allowed."""
    import torch
    T, B, D, H, F = 32, 2, 128, 96, 160
    block = example.Block(D, H, F, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(T, B, D, generator=gen, device="cuda").bfloat16()
    dy = torch.randn(T, B, D, generator=gen, device="cuda")
    state = torch.randn(B, H, generator=gen, device="cuda")
    y, last, kept = block.forward(x, state)
    got = block.backward(dy, kept)
    W = {k: v.double().requires_grad_() for k, v in block.W.items()}
    xd, h, hs = x.double(), state.double(), []
    g = xd @ W["Wg"].T
    for t in range(T):
        z = torch.sigmoid(g[t, :, :H])
        h = z * h + (1 - z) * g[t, :, H:]
        hs.append(h)
    x1 = xd + torch.stack(hs) @ W["Wo"].T
    p = x1 @ W["Wf"].T
    ref = x1 + (torch.nn.functional.silu(p[..., :F]) * p[..., F:]) @ W["Wd"].T
    ref.backward(dy.double())
    assert (y.double() - ref.detach()).norm() <= 0.03 * ref.detach().norm()
    for k, v in got.items():
        assert (v.double() - W[k].grad).norm() <= 0.03 * W[k].grad.norm(), k


def test_serving_equals_the_sequence(example):
    """bf16 activations round at the same places on both sides, but the sums have
    other orders: outputs differ by a few roundings (2^-8) of the largest one."""
    block = example.Block(256, 192, 320, seed=5)
    out, state = example.serve(block)
    assert out <= 4 * 2.0 ** -8 and state <= 4 * 2.0 ** -8
