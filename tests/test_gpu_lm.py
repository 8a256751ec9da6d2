"""The token model: lookup, blocks, loss and optimizer together."""
import pytest
import torch

pytestmark = pytest.mark.gpu

# As for the block alone: a code's uniform error of up to 1.8% of sigma, one such factor in each weight gradient behind it and up to three on the way through a
# block, of which there are two here, and 2^-8 for each bf16 intermediate.
TOL = 0.1


def _reference(net, ids, target, weight):
    """Losses and gradients of the whole model in 64 bits, from its bf16 weights."""
    table = net.weight.double().requires_grad_()
    gamma = net.gamma.double().requires_grad_()
    keep = (ids >= 0) & (ids < table.shape[0])
    x = torch.where(keep[:, None], table[ids.clamp_min(0)] * net.scale, 0.0)
    ws = []
    for b in net.blocks:
        w = {k: v.double().requires_grad_() for k, v in b.weight.items()}
        w["norm"] = b.param["norm"].double().requires_grad_()
        ws.append(w)
        n = x * (x.square().mean(1, keepdim=True) + b.eps).rsqrt() * w["norm"]
        u = n @ w["gate"].t()
        x = x + (u * torch.sigmoid(u) * (n @ w["up"].t())) @ w["down"].t()
    n = x * (x.square().mean(1, keepdim=True) + net.eps).rsqrt() * gamma
    z = n @ table.t()
    has = target >= 0
    loss = torch.where(has, torch.logsumexp(z, 1) - z.gather(1, target.clamp_min(0)[:, None])[:, 0], 0.0)
    (loss * weight.double()).mean().backward()
    return loss.detach(), table.grad, gamma.grad, [{k: v.grad for k, v in w.items()} for w in ws]


@pytest.mark.parametrize("vocab,hidden,ffn,layers,tokens", [(503, 128, 352, 2, 300), (64, 130, 300, 1, 65)])
def test_gradients(vocab, hidden, ffn, layers, tokens):
    from paper_2608_22322_amd.lm import TokenModel

    net = TokenModel(vocab, hidden, ffn, layers, tokens, seed=2)
    g = torch.Generator(device="cuda").manual_seed(3)
    ids = torch.randint(vocab, (tokens,), device="cuda", generator=g)
    target = torch.randint(vocab, (tokens,), device="cuda", generator=g)
    ids[5], target[3::10] = -1, -100
    weight = torch.rand(tokens, device="cuda", generator=g)
    loss = net.gradients(ids, target, weight)
    want, table, gamma, blocks = _reference(net, ids, target, weight)

    def off(a, b):
        return float((a.double() - b).norm() / b.norm())

    assert off(loss, want) < 0.01
    assert off(net.table_grad, table) < TOL and off(net.gamma_grad, gamma) < TOL
    for b, w in zip(net.blocks, blocks):
        for k, v in w.items():
            assert off(b.grad[k], v) < TOL, k


def test_training_runs_and_repeats():
    from paper_2608_22322_amd.lm import train

    runs = [train(vocab=300, hidden=128, ffn=256, layers=2, tokens=200, steps=3) for _ in range(2)]
    (a, la), (b, lb) = runs
    assert la == lb and all(x == x for x in la)
    assert torch.equal(a.table, b.table) and all(torch.equal(x.param[k], y.param[k]) for x, y in zip(a.blocks, b.blocks) for k in x.param)
    assert not torch.equal(a.blocks[0].param["gate"], train(vocab=300, hidden=128, ffn=256, layers=2, tokens=200, steps=1)[0].blocks[0].param["gate"])
