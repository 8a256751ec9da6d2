"""The activation operators together: an MLP block's gradients and its training with 8-bit activations and states."""
import pytest
import torch

pytestmark = pytest.mark.gpu

# A code's step is at most 1/64 of its block's largest value, about 3 to 4 sigma of 64 normal values: a uniform error of
# at most 4 / 64 / sqrt(12) = 1.8% of sigma, one such factor in each weight gradient and up to three on the way
# through the gated activation's derivative; the bf16 intermediates add 2^-8 each. 6% of a gradient's norm covers them.
TOL = 0.06


def _reference(net, x, dy):
    """Gradients of the block in 64 bits, from its bf16 weights."""
    w = {k: v.double().requires_grad_() for k, v in net.weight.items()}
    gamma, x = net.param["norm"].double().requires_grad_(), x.double().requires_grad_()
    n = x * (x.square().mean(1, keepdim=True) + net.eps).rsqrt() * gamma
    a, b = n @ w["gate"].t(), n @ w["up"].t()
    y = x + (a * torch.sigmoid(a) * b) @ w["down"].t()
    y.backward(dy.double())
    return y.detach(), x.grad, {"gate": w["gate"].grad, "up": w["up"].grad, "down": w["down"].grad, "norm": gamma.grad}


@pytest.mark.parametrize("hidden,ffn,tokens,block", [(256, 704, 300, 64), (130, 300, 77, 32), (1024, 2816, 512, 128)])
def test_block_gradients(hidden, ffn, tokens, block):
    from paper_2608_22322_amd.mlp import SwigluMLP

    net = SwigluMLP(hidden, ffn, tokens, block, seed=3)
    g = torch.Generator(device="cuda").manual_seed(5)
    net.param["norm"].add_(torch.empty_like(net.param["norm"]).normal_(0, 0.1, generator=g))
    x = torch.empty(tokens, hidden, device="cuda").normal_(generator=g).bfloat16()
    dy = torch.empty(tokens, hidden, device="cuda").normal_(generator=g).bfloat16()
    y, dx, grads = _reference(net, x, dy)

    def off(a, b):
        return float((a.double() - b).norm() / b.norm())

    assert off(net.forward(x), y) < 2.0**-7  # a bf16 result of bf16 intermediates: the residual keeps it close
    assert off(net.backward(dy), dx) < TOL
    for k, want in grads.items():
        assert off(net.grad[k], want) < TOL, k
    assert net.saved_bytes() < 0.5 * net.bf16_bytes()


def test_training_lowers_the_loss():
    from paper_2608_22322_amd.mlp import train

    _, losses = train(hidden=256, ffn=704, tokens=512, steps=30, lr=3e-3)
    assert losses[-1] < 0.5 * losses[0] and all(b < 1.5 * a for a, b in zip(losses, losses[1:]))


def test_passes_repeat_bit_for_bit():
    from paper_2608_22322_amd.mlp import SwigluMLP

    a, b = SwigluMLP(256, 704, 200, seed=1), SwigluMLP(256, 704, 200, seed=1)
    x = torch.randn(200, 256, device="cuda").bfloat16()
    res = []
    for net in (a, b):
        for t in (1, 2):
            y = net.forward(x)
            dx = net.backward(y)
            net.step(t)
        res.append((y, dx, *net.grad.values(), *net.param.values()))
    assert all(torch.equal(p, q) for p, q in zip(*res))
