"""Activations in 8 bits: the code, the operators that save it and the ones that use it.

A training program keeps each layer's inputs for the backward pass. Here they are kept as E8 codes (a signed byte per
value, one power-of-two step per block of 32, 64 or 128 columns of a row) and the backward pass computes from the codes:

* :func:`quantize`, :func:`dequantize`: the code itself.
* :func:`norm_forward`, :func:`norm_backward`: layer and RMS norm. The code of the normalised input serves the norm's
  backward pass and, with the norm's weight as a scale, the weight gradient of every linear layer that reads its output.
* :func:`swiglu_forward`, :func:`swiglu_backward`: silu(gate) * up from the codes of gate and up; the backward pass
  also gives the code of its output, for the next linear layer's weight gradient.
* :func:`linear_wgrad`: a linear layer's weight (and bias) gradient from its input's code.

Matrices are 2-D tensors of float32 or bfloat16, rows contiguous (any row pitch, so slices of wider buffers will do; rows that
overlap, as those of an expanded row do, are refused).
Every call enqueues on `stream` (default: the current stream) and returns; outputs and workspaces are the caller's. The
operands of a call, its workspace and its stream belong to one GPU, which has to be the current one (`torch.cuda.device`).
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

import torch

from . import DTYPE_BF16, DTYPE_F32, check, lib

LAYER, RMS = 0, 1
BLOCKS = (32, 64, 128)


class _Dtypes(dict):
    def __missing__(self, dtype):
        raise ValueError(f"dtype {dtype}: float32 or bfloat16 is needed")


_DTYPES = _Dtypes({torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16})


@dataclass
class ActCode:
    """The E8 code of a rows x cols matrix: codes int8 [rows, blocks * block], exps uint8 [rows, blocks]."""
    codes: torch.Tensor
    exps: torch.Tensor
    rows: int
    cols: int
    block: int = 64

    def __post_init__(self):
        if self.block not in BLOCKS:
            raise ValueError(f"block {self.block} must be 32, 64 or 128")
        nb = -(-self.cols // self.block)
        for name, t, n, dt in (("codes", self.codes, nb * self.block, torch.int8), ("exps", self.exps, nb, torch.uint8)):
            if t.dtype != dt or not t.is_contiguous() or t.numel() < self.rows * n or not t.is_cuda:
                raise ValueError(f"{name}: a contiguous {dt} GPU tensor of {self.rows} x {n} is needed")

    def nbytes(self) -> int:
        return self.codes.numel() + self.exps.numel()


def code_bytes(rows: int, cols: int, block: int = 64) -> int:
    """Bytes of codes and exponents of a rows x cols matrix."""
    codes, exps = lib().al_act_code_bytes(rows, cols, block), lib().al_act_exp_bytes(rows, cols, block)
    if codes < 0 or exps < 0:
        raise ValueError(f"no code of {rows} x {cols} values in blocks of {block}")
    return codes + exps


def alloc_code(rows: int, cols: int, block: int = 64, device="cuda") -> ActCode:
    nb = -(-cols // block)
    return ActCode(torch.empty(rows, nb * block, dtype=torch.int8, device=device),
                   torch.empty(rows, nb, dtype=torch.uint8, device=device), rows, cols, block)


# ---------------------------------------------------------------------------- argument checks
def _dtype(t) -> int:
    return _DTYPES[t.dtype]


def _gpu(t, stream=None) -> int:
    """The GPU of a call, from its first operand. A kernel runs on the current GPU (or its stream's), whatever its operands' is."""
    dev, now = t.get_device(), torch._C._cuda_getDevice()
    if dev != now:
        raise ValueError(f"operands on cuda:{dev} while cuda:{now} is the current device: call under torch.cuda.device({dev})")
    if stream is not None and getattr(stream, "device_index", dev) != dev:
        raise ValueError(f"operands on cuda:{dev}, the stream on cuda:{stream.device_index}")
    return dev


def _mat(t, name: str, rows: int, cols: int, dtype, dev=None):
    """(pointer, row pitch) of a rows x cols matrix of dtype on GPU `dev` (None: on any); (None, 0) for None."""
    if t is None:
        return None, 0
    if t.dtype is not dtype or t.shape != (rows, cols) or not (t.is_cuda if dev is None else t.get_device() == dev):
        raise ValueError(f"{name}: a {rows} x {cols} {dtype} GPU tensor is needed{_on(dev)}, got {tuple(t.shape)} {t.dtype} on {t.device}")
    ld, inner = t.stride()
    if inner != 1 and cols > 1:
        raise ValueError(f"{name}: rows must be contiguous (strides {t.stride()})")
    return t.data_ptr(), ld if rows > 1 else cols  # the library refuses a pitch below cols


def _on(dev) -> str:
    return "" if dev is None else f" on cuda:{dev}"


def _vec(t, name: str, n: int, dtype, dev: int):
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{name}: a contiguous {dtype} GPU tensor of {n} is needed{_on(dev)}")
    return t.data_ptr()


def _code(c, name: str, rows: int, cols: int, dev: int):
    """(codes, exps, block) of a code that has to be of a rows x cols matrix."""
    if c is None:
        return None, None, 0
    if c.rows != rows or c.cols != cols:
        raise ValueError(f"{name}: the code of a {rows} x {cols} matrix is needed, got {c.rows} x {c.cols}")
    if c.codes.get_device() != dev or c.exps.get_device() != dev:
        raise ValueError(f"{name}: the code is on {c.codes.device} and {c.exps.device}, needed{_on(dev)}")
    return c.codes.data_ptr(), c.exps.data_ptr(), c.block


def _scratch(ws, dev: int):
    """(pointer, bytes) of a workspace; (None, 0) for None."""
    if ws is None:
        return None, 0
    if ws.get_device() != dev or not ws.is_contiguous():
        raise ValueError(f"ws: a contiguous GPU tensor is needed{_on(dev)}, got one on {ws.device}")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _queue(stream, dev: int):
    """The stream's handle; None: the current stream of the GPU (read directly: torch's Stream object takes 2.6 us of
    a 6 us call to build)."""
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(dev)


def _shape(t, name: str):
    if t.dim() != 2:
        raise ValueError(f"{name}: a matrix is needed, got {tuple(t.shape)}")
    return t.shape


# ------------------------------------------------------------------------------------- the code
def quantize(x, code: ActCode, stream=None) -> None:
    """code <- E8 code of x."""
    rows, cols = _shape(x, "x")
    p, ld = _mat(x, "x", rows, cols, x.dtype)
    dev = _gpu(x, stream)
    c, e, block = _code(code, "code", rows, cols, dev)
    check(lib().al_act_quantize(_dtype(x), p, ld, rows, cols, block, c, e, _queue(stream, dev)))


def dequantize(code: ActCode, out, stream=None) -> None:
    """out <- the values of the code (exact in bfloat16)."""
    p, ld = _mat(out, "out", code.rows, code.cols, out.dtype)
    dev = _gpu(out, stream)
    c, e, block = _code(code, "code", code.rows, code.cols, dev)
    check(lib().al_act_dequantize(c, e, code.rows, code.cols, block, _dtype(out), p, ld, _queue(stream, dev)))


# ---------------------------------------------------------------------------------------- norms
def norm_forward(kind: int, x, y, mean=None, rstd=None, gamma=None, beta=None, eps: float = 1e-5,
                 code: ActCode | None = None, stream=None) -> None:
    """y = xhat gamma + beta with xhat = (x - mean) rstd over each row (RMS: mean 0, no beta); writes mean (LAYER)
    and rstd if given, and the code of xhat if `code` is."""
    rows, cols = _shape(x, "x")
    dt = x.dtype
    px, ldx = _mat(x, "x", rows, cols, dt)
    dev = _gpu(x, stream)
    py, ldy = _mat(y, "y", rows, cols, dt, dev)
    f = torch.float32
    c, e, block = _code(code, "code", rows, cols, dev)
    check(lib().al_norm_forward(kind, _dtype(x), px, ldx, rows, cols, eps, _vec(gamma, "gamma", cols, f, dev),
                                _vec(beta, "beta", cols, f, dev), py, ldy, _vec(mean, "mean", rows, f, dev),
                                _vec(rstd, "rstd", rows, f, dev), block, c, e, _queue(stream, dev)))


def norm_backward_workspace_bytes(kind: int, rows: int, cols: int, dtype=torch.bfloat16) -> int:
    out = ctypes.c_size_t(0)
    check(lib().al_norm_backward_workspace_bytes(kind, _DTYPES[dtype], rows, cols, ctypes.byref(out)))
    return out.value


def norm_backward(kind: int, dy, x, mean, rstd, dx, gamma=None, dgamma=None, dbeta=None, add=None, ws=None,
                  stream=None) -> None:
    """Backward pass of norm_forward. x: its input, or the ActCode of xhat (mean is then not needed). dx gets the
    input's gradient plus `add` (may be dx itself); dgamma, dbeta (of one dtype) the weights' gradients."""
    rows, cols = _shape(dy, "dy")
    dt = dy.dtype
    f = torch.float32
    pdy, lddy = _mat(dy, "dy", rows, cols, dt)
    dev = _gpu(dy, stream)
    if isinstance(x, ActCode):
        c, e, block = _code(x, "x", rows, cols, dev)
        px, ldx, mean = None, 0, None
    else:
        c, e, block = None, None, 0
        px, ldx = _mat(x, "x", rows, cols, dt, dev)
    pa, lda = _mat(add, "add", rows, cols, dt, dev)
    pdx, lddx = _mat(dx, "dx", rows, cols, dt, dev)
    g = dgamma if dgamma is not None else dbeta
    gt = f if g is None else g.dtype
    check(lib().al_norm_backward(kind, _dtype(dy), pdy, lddy, px, ldx, _vec(mean, "mean", rows, f, dev),
                                 _vec(rstd, "rstd", rows, f, dev), block, c, e, rows, cols, _vec(gamma, "gamma", cols, f, dev),
                                 pa, lda, pdx, lddx, DTYPE_F32 if g is None else _dtype(g),
                                 _vec(dgamma, "dgamma", cols, gt, dev), _vec(dbeta, "dbeta", cols, gt, dev), *_scratch(ws, dev),
                                 _queue(stream, dev)))


# ---------------------------------------------------------------------------- gated activation
def swiglu_forward(gate, up, h, gate_code: ActCode | None = None, up_code: ActCode | None = None, stream=None) -> None:
    """h = silu(gate) * up; writes the codes of gate and up if given (both or neither)."""
    rows, cols = _shape(gate, "gate")
    dt = gate.dtype
    if (gate_code is None) != (up_code is None):
        raise ValueError("the codes of gate and up go together")
    pg, ldg = _mat(gate, "gate", rows, cols, dt)
    dev = _gpu(gate, stream)
    pu, ldu = _mat(up, "up", rows, cols, dt, dev)
    ph, ldh = _mat(h, "h", rows, cols, dt, dev)
    gc, ge, block = _code(gate_code, "gate_code", rows, cols, dev)
    uc, ue, ub = _code(up_code, "up_code", rows, cols, dev)
    if ub != block:
        raise ValueError("the codes of gate and up need one block")
    check(lib().al_swiglu_forward(_dtype(gate), pg, ldg, pu, ldu, rows, cols, ph, ldh, block, gc, ge, uc, ue,
                                  _queue(stream, dev)))


def swiglu_backward(dh, gate_code: ActCode, up_code: ActCode, dgate, dup, h_code: ActCode | None = None,
                    stream=None) -> None:
    """dgate, dup from dh and the saved codes; writes the code of the recomputed h if `h_code` is given."""
    rows, cols = _shape(dh, "dh")
    dt = dh.dtype
    pd, ldd = _mat(dh, "dh", rows, cols, dt)
    dev = _gpu(dh, stream)
    gc, ge, block = _code(gate_code, "gate_code", rows, cols, dev)
    uc, ue, ub = _code(up_code, "up_code", rows, cols, dev)
    hc, he, hb = _code(h_code, "h_code", rows, cols, dev)
    if ub != block or (h_code is not None and hb != block):
        raise ValueError("the codes need one block")
    pg, ldg = _mat(dgate, "dgate", rows, cols, dt, dev)
    pu, ldu = _mat(dup, "dup", rows, cols, dt, dev)
    check(lib().al_swiglu_backward(_dtype(dh), pd, ldd, rows, cols, block, gc, ge, uc, ue, pg, ldg, pu, ldu, hc, he,
                                   _queue(stream, dev)))


# ------------------------------------------------------------------------------ weight gradient
def linear_wgrad_workspace_bytes(dy, code: ActCode, dw) -> int:
    out = ctypes.c_size_t(0)
    check(lib().al_linear_wgrad_workspace_bytes(_dtype(dy), code.rows, dw.shape[0], code.cols, ctypes.byref(out)))
    return out.value


def linear_wgrad(dy, code: ActCode, dw, ws, gamma=None, beta=None, base=None, dbias=None, stream=None) -> None:
    """dw = dy^T (xhat gamma + beta) + base, xhat the values of `code` (tokens x in_features); dbias = column sums of
    dy. dw, base: contiguous [out_features, in_features] of one dtype, base may be dw (accumulation)."""
    tokens, out = _shape(dy, "dy")
    cols = code.cols
    f = torch.float32
    pdy, lddy = _mat(dy, "dy", tokens, out, dy.dtype)
    dev = _gpu(dy, stream)
    c, e, block = _code(code, "code", tokens, cols, dev)
    if dw.shape != (out, cols):
        raise ValueError(f"dw: {out} x {cols} is needed, got {tuple(dw.shape)}")
    gt = dw.dtype
    check(lib().al_linear_wgrad(_dtype(dy), pdy, lddy, c, e, block, tokens, out, cols, _vec(gamma, "gamma", cols, f, dev),
                                _vec(beta, "beta", cols, f, dev), _dtype(dw), _vec(base, "base", out * cols, gt, dev),
                                _vec(dw, "dw", out * cols, gt, dev), _vec(dbias, "dbias", out, gt, dev), *_scratch(ws, dev),
                                _queue(stream, dev)))
