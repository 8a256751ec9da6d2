"""A transformer's pre-norm MLP block trained with 8-bit activations and 8-bit optimizer states.

    y = x + down(silu(gate(n)) * up(n)),  n = rmsnorm(x) gamma

The forward pass keeps three E8 codes and one float per token: xhat (which serves the norm's backward pass and both
weight gradients behind it), gate and up. The backward pass computes from them; the input of `down` is recomputed as a
code on the way. Products with the weights are the library's; everything else runs in this package's kernels, and the
step is al_adamw_step over the block's parameters.

    python -m paper_2608_22322_amd.mlp [--hidden 2048 --ffn 5632 --tokens 2048 --steps 20]
"""
from __future__ import annotations

import argparse
import functools

import torch

from . import AL8, UF8, ParamState, Spec, activations as act, adamw_cfg, adamw_step, adamw_workspace_bytes, alloc_state
from . import log2_floor_of, tensor_array, workspace

NAMES = ("gate", "up", "down", "norm")


def _on_its_gpu(method):
    """Run a method with the block's GPU as the current device, where this package's kernels run."""

    @functools.wraps(method)
    def run(self, *args):
        with torch.cuda.device(self.device):
            return method(self, *args)

    return run


class SwigluMLP:
    """The block's parameters (fp32, with bf16 copies for the products), their gradients and states, and its buffers
    for batches of `tokens` rows, all on `device`."""

    def __init__(self, hidden: int, ffn: int, tokens: int, block: int = 64, eps: float = 1e-5, lr: float = 1e-3, seed: int = 0,
                 device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.hidden, self.ffn, self.tokens, self.eps = hidden, ffn, tokens, eps
        shapes = {"gate": (ffn, hidden), "up": (ffn, hidden), "down": (hidden, ffn), "norm": (1, hidden)}
        bf16 = dict(dtype=torch.bfloat16, device=device)
        self.param, self.grad, self.weight, self.states = {}, {}, {}, []
        m, v = Spec(UF8, 256), Spec(AL8, 2048, log2_floor_of(1e-16))
        for name in NAMES:
            rows, cols = shapes[name]
            p = torch.ones(rows, cols, device=device) if name == "norm" else (
                torch.empty(rows, cols, device=device).normal_(0.0, cols**-0.5, generator=g))
            self.param[name], self.grad[name] = p, torch.zeros(rows, cols, **bf16)
            if name != "norm":
                self.weight[name] = p.bfloat16()
            (mc, mm), (vc, vm) = alloc_state(p.numel(), m, device), alloc_state(p.numel(), v, device)
            self.states.append(ParamState(p, self.grad[name], rows, cols, m=mc, m_meta=mm, v=vc, v_meta=vm))
        self.cfg, self.arr = adamw_cfg(lr=lr, m=m, v=v), tensor_array(self.states)
        self.step_ws = workspace(adamw_workspace_bytes(self.states, self.cfg, arr=self.arr), device)
        # what a batch leaves for its backward pass
        self.xhat = act.alloc_code(tokens, hidden, block, device)
        self.gate_code, self.up_code = act.alloc_code(tokens, ffn, block, device), act.alloc_code(tokens, ffn, block, device)
        self.rstd = torch.empty(tokens, device=device)
        self.device = self.rstd.device
        # scratch of either pass
        self.h_code = act.alloc_code(tokens, ffn, block, device)
        self.n = torch.empty(tokens, hidden, **bf16)
        self.a, self.b, self.h = (torch.empty(tokens, ffn, **bf16) for _ in range(3))
        wide, narrow = act.linear_wgrad_workspace_bytes, act.norm_backward_workspace_bytes
        self.ws = workspace(max(wide(self.a, self.xhat, self.grad["gate"]), wide(self.n, self.h_code, self.grad["down"]),
                                narrow(act.RMS, tokens, hidden)), device)

    def saved_bytes(self) -> int:
        """Bytes that a batch keeps between its forward and its backward pass."""
        return self.xhat.nbytes() + self.gate_code.nbytes() + self.up_code.nbytes() + 4 * self.tokens

    def bf16_bytes(self, recompute: bool = False) -> int:
        """What a pass in bf16 keeps: x, n, gate, up and h; with `recompute` (as here, n and h again in the backward pass) x, gate
        and up."""
        kept = self.hidden + 2 * self.ffn + (0 if recompute else self.hidden + self.ffn)
        return 2 * self.tokens * kept + 4 * self.tokens

    @_on_its_gpu
    def forward(self, x):
        """y for a [tokens, hidden] bf16 batch."""
        act.norm_forward(act.RMS, x, self.n, rstd=self.rstd, gamma=self.param["norm"].view(-1), eps=self.eps, code=self.xhat)
        torch.mm(self.n, self.weight["gate"].t(), out=self.a)
        torch.mm(self.n, self.weight["up"].t(), out=self.b)
        act.swiglu_forward(self.a, self.b, self.h, self.gate_code, self.up_code)
        return torch.addmm(x, self.h, self.weight["down"].t())

    @_on_its_gpu
    def backward(self, dy):
        """dx from dy, the parameters' gradients into self.grad (what the last forward pass saved is used)."""
        gamma = self.param["norm"].view(-1)
        torch.mm(dy, self.weight["down"], out=self.h)  # dh
        act.swiglu_backward(self.h, self.gate_code, self.up_code, self.a, self.b, h_code=self.h_code)
        act.linear_wgrad(dy, self.h_code, self.grad["down"], self.ws)
        act.linear_wgrad(self.a, self.xhat, self.grad["gate"], self.ws, gamma=gamma)
        act.linear_wgrad(self.b, self.xhat, self.grad["up"], self.ws, gamma=gamma)
        torch.mm(self.a, self.weight["gate"], out=self.n)  # dn
        torch.addmm(self.n, self.b, self.weight["up"], out=self.n)
        dx = torch.empty_like(dy)
        act.norm_backward(act.RMS, self.n, self.xhat, None, self.rstd, dx, gamma=gamma, dgamma=self.grad["norm"].view(-1), add=dy,
                          ws=self.ws)
        return dx

    @_on_its_gpu
    def step(self, t: int) -> None:
        """One AdamW step (8-bit states) and the weights' bf16 copies from the new parameters."""
        adamw_step(self.states, self.cfg, t, self.step_ws, arr=self.arr)
        for name, w in self.weight.items():
            w.copy_(self.param[name])


def train(hidden=2048, ffn=5632, tokens=2048, steps=20, block=64, lr=1e-3, seed=0):
    """Fit a block to the outputs of another one on random batches; returns the block and the loss of each step."""
    net, teacher = SwigluMLP(hidden, ffn, tokens, block, lr=lr, seed=seed), SwigluMLP(hidden, ffn, tokens, block, seed=seed + 1)
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    x = torch.empty(tokens, hidden, device="cuda").normal_(generator=g).bfloat16()
    want = teacher.forward(x).float()
    losses = []
    for t in range(1, steps + 1):
        off = net.forward(x).float() - want
        losses.append(float(off.square().mean()))
        net.backward((off * (2.0 / off.shape[0])).bfloat16())
        net.step(t)
    return net, losses


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("hidden", 2048), ("ffn", 5632), ("tokens", 2048), ("steps", 20), ("block", 64)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    net, losses = train(a.hidden, a.ffn, a.tokens, a.steps, a.block)
    print("saved for the backward pass: %.1f MiB (in bf16 %.1f MiB with the same recomputation, %.1f MiB without)"
          % tuple(n / 2**20 for n in (net.saved_bytes(), net.bf16_bytes(recompute=True), net.bf16_bytes())))
    print("loss: %.5f -> %.5f in %d steps" % (losses[0], losses[-1], len(losses)))


if __name__ == "__main__":
    main()
