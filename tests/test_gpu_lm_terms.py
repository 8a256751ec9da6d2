"""The two terms of a tied table's gradient, each by itself: the head's and the lookup's."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TOL = 0.1  # the blocks' 8-bit codes, as for the whole model


@pytest.mark.parametrize("vocab,hidden,ffn,layers,tokens", [(503, 128, 352, 2, 300), (4001, 136, 300, 1, 65), (97, 64, 128, 0, 50)])
def test_both_uses_of_the_table(vocab, hidden, ffn, layers, tokens):
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import vocab as voc
    from paper_2608_22322_amd.lm import TokenModel

    net = TokenModel(vocab, hidden, ffn, layers, tokens, seed=5)
    g = torch.Generator(device="cuda").manual_seed(6)
    ids, target = (torch.randint(vocab, (tokens,), device="cuda", generator=g) for _ in range(2))
    weight = torch.rand(tokens, device="cuda", generator=g)
    net.gradients(ids, target, weight=weight)

    table, head = (net.weight.double().requires_grad_() for _ in range(2))
    x = table[ids] * net.scale
    for b in net.blocks:
        n = x * (x.square().mean(1, keepdim=True) + b.eps).rsqrt() * b.param["norm"].double()
        u = n @ b.weight["gate"].double().t()
        x = x + (u * torch.sigmoid(u) * (n @ b.weight["up"].double().t())) @ b.weight["down"].double().t()
    z = (x * (x.square().mean(1, keepdim=True) + net.eps).rsqrt() * net.gamma.double()) @ head.t()
    ((torch.logsumexp(z, 1) - z.gather(1, target[:, None])[:, 0]) * weight.double()).mean().backward()

    # the head's term from its own inputs, and the lookup's as the rest: the sum was rounded to bf16 twice
    dw = torch.empty(vocab, hidden, device="cuda")
    voc.linear_xent(net.n, net.weight, target, None, al.workspace(voc.linear_xent_workspace_bytes(net.n, net.weight, None, dw)), weight=weight, scale=1.0 / tokens, dw=dw)
    assert float((dw.double() - head.grad).norm()) < TOL * float(head.grad.norm())
    rest = net.table_grad.double() - dw.double()
    assert float((rest - table.grad).norm()) < TOL * float(table.grad.norm()) + 2 * 2.0**-8 * float(net.table_grad.double().norm())
    assert 2 * 2.0**-8 * float(net.table_grad.double().norm()) < 0.5 * float(table.grad.norm())  # (a missing term would show)
