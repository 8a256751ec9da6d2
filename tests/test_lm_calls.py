"""Methods of the token model and its blocks take their arguments by position and by name."""
import contextlib

import pytest
import torch


def test_named_arguments_reach_a_method_on_its_gpu(monkeypatch):
    from paper_2608_22322_amd.mlp import _on_its_gpu

    entered = []
    monkeypatch.setattr(torch.cuda, "device", lambda d: entered.append(d) or contextlib.nullcontext())

    class Net:
        device = "cuda:1"

        @_on_its_gpu
        def gradients(self, ids, target, weight=None):
            return ids, target, weight

    assert Net().gradients(1, 2) == (1, 2, None) and Net().gradients(1, 2, 3) == (1, 2, 3)
    assert Net().gradients(1, target=2, weight=3) == (1, 2, 3)
    assert entered == ["cuda:1"] * 3


@pytest.mark.gpu
def test_weights_by_name():
    from paper_2608_22322_amd.lm import TokenModel

    net = TokenModel(64, 64, 128, 1, 30)
    g = torch.Generator(device="cuda").manual_seed(1)
    ids, target = (torch.randint(64, (30,), device="cuda", generator=g) for _ in range(2))
    weight = torch.rand(30, device="cuda", generator=g)
    net.gradients(ids, target, weight)
    want = net.table_grad.clone()
    net.gradients(ids, target=target, weight=weight)
    assert torch.equal(net.table_grad, want)
    net.gradients(ids, target)
    assert not torch.equal(net.table_grad, want)
