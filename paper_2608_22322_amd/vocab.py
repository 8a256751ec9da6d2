"""The two ends of a token model: embeddings and their gradient, and softmax cross entropy of a linear head.

* :func:`embed_forward`, :func:`embed_backward`: the lookup with its scale, and the table's gradient summed over the tokens sorted by id.
* :func:`linear_xent`: each token's loss from the hidden state and the head's weight, and the gradients of both, without the logits in memory.

With a tied table the head's gradient is the lookup's `base` (and its `dw`, in place). A token id or target outside the vocabulary (-100, say) stands for
no token. Matrices, streams, workspaces and devices as in :mod:`.activations`; ids and targets are contiguous int32 or int64 vectors.
"""
from __future__ import annotations

import ctypes

import torch

from . import DTYPE_F32, check, lib
from .activations import _dtype, _gpu, _mat, _on, _queue, _scratch, _shape, _vec

INDEX = {torch.int32: 0, torch.int64: 1}


def _ids(t, name: str, n: int, dev: int):
    if t.dtype not in INDEX or t.numel() != n or t.dim() != 1 or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{name}: a contiguous int32 or int64 GPU vector of {n} is needed{_on(dev)}, got {tuple(t.shape)} {t.dtype} on {t.device}")
    return INDEX[t.dtype], t.data_ptr()


def _packed(t, name: str, rows: int, cols: int, dtype, dev: int):
    if t is None:
        return None
    if t.shape != (rows, cols):
        raise ValueError(f"{name}: {rows} x {cols} is needed, got {tuple(t.shape)}")
    return _vec(t, name, rows * cols, dtype, dev)


def embed_forward(table, ids, out, scale: float = 1.0, stream=None) -> None:
    """out[t] = scale * table[ids[t]] (float32 or bfloat16 each, any row pitch)."""
    vocab, cols = _shape(table, "table")
    tokens, _ = _shape(out, "out")
    pt, ldt = _mat(table, "table", vocab, cols, table.dtype)
    dev = _gpu(table, stream)
    po, ldo = _mat(out, "out", tokens, cols, out.dtype, dev)
    kind, pi = _ids(ids, "ids", tokens, dev)
    check(lib().al_embed_forward(_dtype(table), pt, ldt, vocab, cols, kind, pi, tokens, scale, _dtype(out), po, ldo, _queue(stream, dev)))


def embed_backward_workspace_bytes(dy, dw) -> int:
    out = ctypes.c_size_t(0)
    check(lib().al_embed_backward_workspace_bytes(dy.shape[0], dw.shape[0], dw.shape[1], ctypes.byref(out)))
    return out.value


def embed_backward(dy, ids, dw, ws, scale: float = 1.0, base=None, stream=None) -> None:
    """dw[v] = base[v] + scale * the sum of dy[t] over ids[t] = v. dw, base: contiguous [vocab, cols] of one dtype; base may be dw (rows without a token
    are then not touched)."""
    tokens, cols = _shape(dy, "dy")
    vocab, _ = _shape(dw, "dw")
    pdy, lddy = _mat(dy, "dy", tokens, cols, dy.dtype)
    dev = _gpu(dy, stream)
    kind, pi = _ids(ids, "ids", tokens, dev)
    check(lib().al_embed_backward(_dtype(dy), pdy, lddy, kind, pi, tokens, vocab, cols, scale, _dtype(dw),
                                  _packed(base, "base", vocab, cols, dw.dtype, dev), _packed(dw, "dw", vocab, cols, dw.dtype, dev), *_scratch(ws, dev),
                                  _queue(stream, dev)))


def _kind(t) -> int:
    return DTYPE_F32 if t is None else _dtype(t)


def linear_xent_workspace_bytes(h, w, dh=None, dw=None) -> int:
    tokens, hidden = _shape(h, "h")
    vocab, _ = _shape(w, "w")
    out = ctypes.c_size_t(0)
    check(lib().al_linear_xent_workspace_bytes(tokens, hidden, vocab, w.stride(0) if vocab > 1 else hidden, dh is not None, _kind(dh), dw is not None, _kind(dw),
                                               ctypes.byref(out)))
    return out.value


def linear_xent(h, w, target, loss, ws, weight=None, scale: float = 1.0, lse=None, dh=None, dw=None, base=None, stream=None) -> None:
    """loss[t] = logsumexp(h[t] w^T) - (h[t] w^T)[target[t]] for bfloat16 h [tokens, hidden] and w [vocab, hidden] (0 without a target), and the gradients of
    scale * sum(weight * loss): dh, dw (+ base), each where it is given. loss, lse, weight: float32 vectors; loss may be None."""
    tokens, hidden = _shape(h, "h")
    vocab, _ = _shape(w, "w")
    f, b = torch.float32, torch.bfloat16
    ph, ldh = _mat(h, "h", tokens, hidden, b)
    dev = _gpu(h, stream)
    pw, ldw = _mat(w, "w", vocab, hidden, b, dev)
    kind, pt = _ids(target, "target", tokens, dev)
    pdh, lddh = _mat(dh, "dh", tokens, hidden, f if dh is None else dh.dtype, dev)
    gt = f if dw is None else dw.dtype
    check(lib().al_linear_xent(ph, ldh, pw, ldw, tokens, hidden, vocab, kind, pt, _vec(weight, "weight", tokens, f, dev), scale,
                               _vec(loss, "loss", tokens, f, dev), _vec(lse, "lse", tokens, f, dev), _kind(dh), pdh, lddh, _kind(dw),
                               _packed(base, "base", vocab, hidden, gt, dev), _packed(dw, "dw", vocab, hidden, gt, dev), *_scratch(ws, dev),
                               _queue(stream, dev)))
