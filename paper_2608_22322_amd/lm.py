"""A small token model trained from its ids to its loss: tied embeddings, pre-norm MLP blocks, cross entropy over the vocabulary.

    x = scale table[ids],  x <- block(x) ...,  loss = cross entropy of rmsnorm(x) gamma against table^T

The blocks are those of :mod:`.mlp` (8-bit activations). The loss and the gradients of its input and of the table come from one call, without logits in
memory; the lookup's gradient is added to the table's in place. Matrices of the blocks take the orthogonalised momentum step, the table and the norms AdamW
(:class:`.muon.MuonStep`), all with 8-bit momentum.

    python -m paper_2608_22322_amd.lm [--vocab 32000 --hidden 2048 --ffn 5632 --layers 2 --tokens 2048 --steps 20]
"""
from __future__ import annotations

import argparse
import math

import torch

from . import ParamState, activations as act, adamw_cfg, muon_cfg, vocab as voc, workspace
from .mlp import SwigluMLP, _on_its_gpu
from .muon import MuonStep


class TokenModel:
    """Parameters (fp32, bf16 copies for the products), gradients (bf16), states and buffers for batches of `tokens` ids, all on `device`."""

    def __init__(self, vocab: int, hidden: int, ffn: int, layers: int, tokens: int, block: int = 64, eps: float = 1e-5, lr: float = 1e-3, seed: int = 0,
                 device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.hidden, self.eps, self.scale = hidden, eps, math.sqrt(hidden)
        self.table = torch.empty(vocab, hidden, device=device).normal_(0.0, 1.0 / self.scale, generator=g)
        self.gamma = torch.ones(1, hidden, device=device)
        self.weight = self.table.bfloat16()
        self.device = self.weight.device
        bf16 = dict(dtype=torch.bfloat16, device=device)
        self.table_grad, self.gamma_grad = torch.zeros(vocab, hidden, **bf16), torch.zeros(1, hidden, **bf16)
        self.blocks = [SwigluMLP(hidden, ffn, tokens, block, eps, None, seed + 1 + i, device) for i in range(layers)]
        self.x, self.n, self.dn = (torch.empty(tokens, hidden, **bf16) for _ in range(3))
        self.code, self.rstd = act.alloc_code(tokens, hidden, block, device), torch.empty(tokens, device=device)
        self.loss = torch.empty(tokens, device=device)
        self.ws = workspace(max(voc.linear_xent_workspace_bytes(self.n, self.weight, self.dn, self.table_grad),
                                voc.embed_backward_workspace_bytes(self.dn, self.table_grad),
                                act.norm_backward_workspace_bytes(act.RMS, tokens, hidden)), device)
        states, names = [ParamState(self.table, self.table_grad, vocab, hidden), ParamState(self.gamma, self.gamma_grad, 1, hidden)], ["embed", "norm"]
        for i, b in enumerate(self.blocks):
            states += b.states
            names += [f"layer{i}.{k}" for k in ("gate", "up", "down", "norm")]
        self.optimizer = MuonStep(states, names, muon_cfg(lr=lr), adamw_cfg(lr=lr), device)

    @_on_its_gpu
    def gradients(self, ids, target, weight=None):
        """Each token's loss, and the gradients of their mean (or of the mean of weight * loss) into the grad buffers."""
        x = self.x
        voc.embed_forward(self.weight, ids, x, self.scale)
        for b in self.blocks:
            x = b.forward(x)
        gamma = self.gamma.view(-1)
        act.norm_forward(act.RMS, x, self.n, rstd=self.rstd, gamma=gamma, eps=self.eps, code=self.code)
        voc.linear_xent(self.n, self.weight, target, self.loss, self.ws, weight=weight, scale=1.0 / target.numel(), dh=self.dn, dw=self.table_grad)
        dx = torch.empty_like(self.dn)
        act.norm_backward(act.RMS, self.dn, self.code, None, self.rstd, dx, gamma=gamma, dgamma=self.gamma_grad.view(-1), ws=self.ws)
        for b in reversed(self.blocks):
            dx = b.backward(dx)
        voc.embed_backward(dx, ids, self.table_grad, self.ws, self.scale, base=self.table_grad)
        return self.loss

    @_on_its_gpu
    def step(self, t: int) -> None:
        """One step of all parameters, and their bf16 copies from them."""
        self.optimizer.step(t)
        self.weight.copy_(self.table)
        for b in self.blocks:
            b.refresh()


def train(vocab=32000, hidden=2048, ffn=5632, layers=2, tokens=2048, steps=20, lr=1e-3, seed=0):
    """Learn a fixed successor of every id on random batches; returns the model and the mean loss of each step."""
    net = TokenModel(vocab, hidden, ffn, layers, tokens, lr=lr, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 99)
    successor = torch.randperm(vocab, device="cuda", generator=g)
    losses = []
    for t in range(1, steps + 1):
        ids = torch.randint(vocab, (tokens,), device="cuda", generator=g)
        losses.append(float(net.gradients(ids, successor[ids]).mean()))
        net.step(t)
    return net, losses


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("vocab", 32000), ("hidden", 2048), ("ffn", 5632), ("layers", 2), ("tokens", 2048), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    _, losses = train(a.vocab, a.hidden, a.ffn, a.layers, a.tokens, a.steps)
    print("loss: %.5f -> %.5f in %d steps" % (losses[0], losses[-1], len(losses)))


if __name__ == "__main__":
    main()
