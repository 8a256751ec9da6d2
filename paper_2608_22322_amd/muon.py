"""Orthogonalised updates: the Newton-Schulz products by themselves, and the step of a model whose matrices take them.

Which tensors: the 2-D weights of the transformer blocks, those that APOLLO projects. The token embedding, the LM head and 1-D tensors
keep AdamW with the same momentum code. A matrix then holds one state, its momentum (8 bits and a float per 256 elements in UF8).
"""
from __future__ import annotations

import ctypes

import torch

from . import ORTHO_COEFS, check, lib, ortho_cfg
from .activations import _dtype, _gpu, _mat, _queue, _scratch, _shape
from .apollo import projected as orthogonalised

__all__ = ("MuonStep", "orthogonalize", "orthogonalize_workspace_bytes", "orthogonalised")


def _parts(out, parts):
    return parts if parts is not None else 2 if out.dtype is torch.float32 else 1


def orthogonalize_workspace_bytes(x, out, parts: int | None = None) -> int:
    rows, cols = _shape(x, "x")
    n = ctypes.c_size_t(0)
    check(lib().al_orthogonalize_workspace_bytes(rows, cols, ctypes.byref(ortho_cfg(parts=_parts(out, parts))), ctypes.byref(n)))
    return n.value


def orthogonalize(x, out, ws, steps: int = 5, coefs=ORTHO_COEFS, eps: float = 1e-7, parts: int | None = None, stream=None) -> None:
    """out <- x with its singular values taken to about 1 by `steps` Newton-Schulz steps (out may be x).

    x, out: float32 or bfloat16 matrices of any row pitch. parts: 1 holds the matrices between the products in 11 bits (the default for a bfloat16 out), 2 in
    22 (the default for a float32 out). ws: orthogonalize_workspace_bytes(x, out, parts) bytes."""
    rows, cols = _shape(x, "x")
    px, ldx = _mat(x, "x", rows, cols, x.dtype)
    dev = _gpu(x, stream)
    po, ldo = _mat(out, "out", rows, cols, out.dtype, dev)
    cfg = ortho_cfg(steps, coefs, eps, _parts(out, parts))
    check(lib().al_orthogonalize(_dtype(x), px, ldx, rows, cols, ctypes.byref(cfg), _dtype(out), po, ldo, *_scratch(ws, dev), _queue(stream, dev)))


class MuonStep:
    """One step per call over a list of ParamState (param, grad, rows, cols) with names: block matrices take al_muon_step, the others al_adamw_step
    (states allocated here, the momentum by `cfg.m`). Matrices share launches, and the roundings of one's update go with the list: processes that have to agree bit for bit step the same list."""

    def __init__(self, states, names, cfg=None, adamw=None, device="cuda"):
        from . import (Spec, adamw_cfg, adamw_workspace_bytes, alloc_state, muon_cfg, muon_workspace_bytes, tensor_array, workspace)

        self.cfg = cfg or muon_cfg()
        m = Spec(self.cfg.m.codec, self.cfg.m.block, self.cfg.m.log_floor)
        self.full_cfg = adamw or adamw_cfg(lr=self.cfg.lr, weight_decay=self.cfg.weight_decay, grad_bf16=self.cfg.grad_dtype == 1, m=m)
        v = Spec(self.full_cfg.v.codec, self.full_cfg.v.block, self.full_cfg.v.log_floor)
        fm = Spec(self.full_cfg.m.codec, self.full_cfg.m.block, self.full_cfg.m.log_floor)
        self.ortho_states, self.full_states = [], []
        for st, name in zip(states, names):
            n = st.rows * st.cols
            if orthogonalised(name, st.rows, st.cols):
                st.m, st.m_meta = alloc_state(n, m, device)
                self.ortho_states.append(st)
            else:
                st.m, st.m_meta = alloc_state(n, fm, device)
                st.v, st.v_meta = alloc_state(n, v, device)
                self.full_states.append(st)
        self.arr, self.full_arr = tensor_array(self.ortho_states), tensor_array(self.full_states)
        self.ws = workspace(muon_workspace_bytes(self.ortho_states, self.cfg, arr=self.arr), device)
        self.full_ws = workspace(adamw_workspace_bytes(self.full_states, self.full_cfg, arr=self.full_arr), device)

    def step(self, t: int, stream=None) -> None:
        from . import adamw_step, muon_step

        muon_step(self.ortho_states, self.cfg, t, self.ws, stream=stream, arr=self.arr)
        if self.full_states:
            adamw_step(self.full_states, self.full_cfg, t, self.full_ws, stream=stream, arr=self.full_arr)
