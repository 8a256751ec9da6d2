"""CPU tests of the activation operators' C ABI: refusals before any HIP call, sizes, and the code's definition."""
import ctypes

import numpy as np
import pytest

import paper_2608_22322_amd as al
from tests.act_util import decode, encode

A = 1 << 20  # a 16-byte aligned fake device address (never dereferenced: validation fails first)


def _status(fn, *args):
    return getattr(al.lib(), fn)(*args)


def test_sizes():
    L = al.lib()
    assert L.al_act_code_bytes(3, 100, 64) == 3 * 128 and L.al_act_exp_bytes(3, 100, 64) == 3 * 2
    assert L.al_act_code_bytes(3, 0, 64) == 0 and L.al_act_exp_bytes(0, 5, 128) == 0
    for bad in ((-1, 5, 64), (5, -1, 64), (5, 5, 16), (5, 5, 256)):
        assert L.al_act_code_bytes(*bad) == -1 and L.al_act_exp_bytes(*bad) == -1


def test_the_code_is_within_a_step():
    """The definition itself: half a step of the block's power of two, one at the ends; a step is a / 128 to a / 64."""
    rng = np.random.default_rng(0)
    x = (rng.normal(size=(200, 300)) * np.exp2(rng.integers(-60, 60, (200, 1)))).astype(np.float32)
    for block in (32, 64, 128):
        codes, exps = encode(x, block)
        step = np.ldexp(1.0, exps.astype(int) - 127).repeat(block, 1)[:, :300]
        ends = np.abs(codes[:, :300].astype(int)) == 127
        assert (np.abs(decode(codes, exps, 300, block) - x) <= np.where(ends, 1.0, 0.5) * step).all()
        v = np.zeros((200, exps.shape[1] * block))
        v[:, :300] = np.abs(x)
        top = v.reshape(200, -1, block).max(-1)
        s = np.ldexp(1.0, exps.astype(int) - 127)
        assert (s * 64 <= top).all() and (top < s * 128).all()
        got = decode(codes, exps, 300, block)
        assert np.array_equal(got, got.astype(np.float32))  # and in bf16: 7 bits and a sign
        assert np.array_equal(np.frexp(got)[0] * 128, np.rint(np.frexp(got)[0] * 128))


def _quantize(dtype=1, x=A, ld=100, rows=8, cols=100, block=64, codes=A, exps=A):
    return _status("al_act_quantize", dtype, x, ld, rows, cols, block, codes, exps, None)


def _dequantize(codes=A, exps=A, rows=8, cols=100, block=64, dtype=1, out=A, ld=100):
    return _status("al_act_dequantize", codes, exps, rows, cols, block, dtype, out, ld, None)


@pytest.mark.parametrize("call", [_quantize, _dequantize])
def test_code_refusals(call):
    assert call(dtype=2) == 1 and call(rows=-1) == 1 and call(block=16) == 1 and call(ld=99) == 1
    assert call(codes=None) == 1 and call(exps=None) == 1 and call(codes=A + 8) == 2 and call(exps=A + 1) == 2
    data = "x" if call is _quantize else "out"
    assert call(**{data: None}) == 1 and call(**{data: A + 1}) == 2 and call(**{data: A + 2, "dtype": 0}) == 2
    assert call(rows=1 << 31) == 4 and call(ld=1 << 46) == 4
    assert call(rows=0) == 0 and call(cols=0) == 0  # nothing to do, no HIP call
    assert "al_act" in (call(block=7), al.lib().al_last_error().decode())[1]


def _forward(kind=0, dtype=1, x=A, ldx=100, rows=8, cols=100, eps=1e-5, gamma=A, beta=A, y=2 * A, ldy=100, mean=A, rstd=A, block=64,
             codes=None, exps=None):
    return _status("al_norm_forward", kind, dtype, x, ldx, rows, cols, eps, gamma, beta, y, ldy, mean, rstd, block, codes, exps, None)


def test_norm_forward_refusals():
    assert _forward(kind=2) == 1 and _forward(dtype=9) == 1 and _forward(cols=-1) == 1 and _forward(eps=float("nan")) == 1
    assert _forward(eps=-1e-9) == 1 and _forward(x=None) == 1 and _forward(y=None) == 1 and _forward(ldy=50) == 1
    assert _forward(kind=1) == 1 and _forward(kind=1, beta=None) == 1  # RMS: neither beta nor mean
    assert _forward(y=A, ldy=104) == 1  # in place with another pitch
    assert _forward(gamma=A + 2) == 2 and _forward(rstd=A + 1) == 2 and _forward(y=A + 1) == 2
    assert _forward(codes=A) == 1 and _forward(exps=A) == 1 and _forward(codes=A, exps=A, block=48) == 1
    assert _forward(codes=A + 4, exps=A) == 2
    assert _forward(rows=0) == 0 and _forward(cols=0) == 0


def _backward(kind=0, dtype=1, dy=A, lddy=100, x=2 * A, ldx=100, mean=A, rstd=A, block=64, codes=None, exps=None, rows=8, cols=100,
              gamma=A, add=None, ldadd=0, dx=3 * A, lddx=100, grad_dtype=0, dgamma=A, dbeta=A, ws=A, ws_bytes=1 << 30):
    return _status("al_norm_backward", kind, dtype, dy, lddy, x, ldx, mean, rstd, block, codes, exps, rows, cols, gamma, add, ldadd, dx,
                   lddx, grad_dtype, dgamma, dbeta, ws, ws_bytes, None)


def test_norm_backward_refusals():
    need = ctypes.c_size_t(0)
    assert _status("al_norm_backward_workspace_bytes", 0, 1, 8, 100, ctypes.byref(need)) == 0 and need.value > 0
    assert _status("al_norm_backward_workspace_bytes", 0, 1, 8, 100, None) == 1
    assert _status("al_norm_backward_workspace_bytes", 3, 1, 8, 100, ctypes.byref(need)) == 1
    assert _status("al_norm_backward_workspace_bytes", 0, 1, 8, 100, ctypes.byref(need)) == 0
    assert _backward(ws=None) == 3 and _backward(ws_bytes=need.value - 1) == 3 and _backward(ws=A + 64) == 2
    assert _backward(kind=5) == 1 and _backward(grad_dtype=3) == 1 and _backward(rows=-2) == 1
    assert _backward(kind=1, mean=None) == 1 and _backward(kind=1, dbeta=None) == 1  # RMS: neither
    assert _backward(mean=None) == 1 and _backward(rstd=None) == 1 and _backward(dy=None) == 1 and _backward(dx=None) == 1
    assert _backward(x=None) == 1 and _backward(codes=A, exps=A) == 1 and _backward(codes=A, exps=A, x=None) == 1  # mean with a code
    assert _backward(codes=A, exps=A, x=None, mean=None, block=40) == 1
    assert _backward(dx=A) == 1 and _backward(dx=2 * A) == 1 and _backward(add=3 * A, ldadd=104) == 1
    assert _backward(dgamma=A + 1) == 2 and _backward(dgamma=A + 2) == 2 and _backward(add=A + 1, ldadd=100) == 2


def test_swiglu_refusals():
    def f(dtype=1, gate=A, ldg=100, up=A, ldu=100, rows=8, cols=100, h=A, ldh=100, block=64, gc=A, ge=A, uc=A, ue=A):
        return _status("al_swiglu_forward", dtype, gate, ldg, up, ldu, rows, cols, h, ldh, block, gc, ge, uc, ue, None)

    def b(dtype=1, dh=A, ld=100, rows=8, cols=100, block=64, gc=A, ge=A, uc=A, ue=A, dg=A, ldg=100, du=A, ldu=100, hc=A, he=A):
        return _status("al_swiglu_backward", dtype, dh, ld, rows, cols, block, gc, ge, uc, ue, dg, ldg, du, ldu, hc, he, None)

    for call in (f, b):
        assert call(dtype=5) == 1 and call(rows=-1) == 1 and call(block=96) == 1 and call(gc=None) == 1 and call(ue=None) == 1
        assert call(uc=A + 8) == 2 and call(ldg=99) == 1 and call(ldu=99) == 1 and call(rows=0) == 0 and call(cols=0) == 0
    assert f(gate=None) == 1 and f(up=A + 1) == 2 and f(h=None) == 1
    assert b(dh=None) == 1 and b(dg=None) == 1 and b(du=A + 1) == 2 and b(he=None) == 1 and b(hc=A + 4) == 2


def test_wgrad_refusals():
    def w(dtype=1, dy=A, ld=100, codes=A, exps=A, block=64, tokens=64, out=100, cols=200, gamma=A, beta=A, gt=0, base=A, dw=A, db=A, ws=A,
          wb=1 << 40):
        return _status("al_linear_wgrad", dtype, dy, ld, codes, exps, block, tokens, out, cols, gamma, beta, gt, base, dw, db, ws, wb, None)

    need = ctypes.c_size_t(0)
    assert _status("al_linear_wgrad_workspace_bytes", 1, 64, 100, 200, ctypes.byref(need)) == 0 and need.value > 0
    assert _status("al_linear_wgrad_workspace_bytes", 1, 64, 100, 200, None) == 1
    assert _status("al_linear_wgrad_workspace_bytes", 1, -1, 100, 200, ctypes.byref(need)) == 1
    assert w(wb=need.value * 0 + 128) == 3 and w(ws=None) == 3 and w(ws=A + 16) == 2
    assert w(dtype=4) == 1 and w(gt=4) == 1 and w(block=256) == 1 and w(tokens=-1) == 1 and w(dy=None) == 1 and w(ld=99) == 1
    assert w(dw=None) == 1 and w(codes=None) == 1 and w(exps=A + 1) == 2 and w(dw=A + 4) == 2 and w(base=A + 8) == 2
    assert w(dy=A + 1) == 2 and w(gamma=A + 1) == 2 and w(db=A + 2) == 2
    assert w(out=(1 << 22) + 1, ld=1 << 23) == 4
    assert w(out=0) == 0


def test_wgrad_sizes_past_the_grids():
    need = ctypes.c_size_t(0)
    for out, cols, want in ((1 << 22, 8, 4), ((1 << 22) - 1, 8, 0), (8, 1 << 29, 4), (8, (1 << 29) - 1, 0)):
        assert _status("al_linear_wgrad_workspace_bytes", 1, 64, out, cols, ctypes.byref(need)) == want
    # splits only where outputs are few: the workspace of a large product is the bias sums alone
    assert _status("al_linear_wgrad_workspace_bytes", 1, 8192, 11008, 4096, ctypes.byref(need)) == 0
    assert need.value <= 11008 * 4 * 257 + 256
    assert _status("al_linear_wgrad_workspace_bytes", 1, 8192, 256, 256, ctypes.byref(need)) == 0
    assert need.value <= 64 << 20


@pytest.mark.parametrize("rows,cols,strides,pitch", [
    (8, 100, (0, 1), 0), (8, 100, (1, 1), 1), (8, 100, (99, 1), 99), (8, 1, (0, 5), 0),  # expanded or overlapping rows keep their pitch
    (8, 100, (100, 1), 100), (8, 100, (107, 1), 107), (1, 100, (0, 1), 100), (0, 100, (100, 1), 100),
])
def test_row_pitch_of_a_tensor(rows, cols, strides, pitch):
    """An expanded row (the gradient of a sum, say) holds one row: taken for a packed matrix it would be read past its end. Its pitch
    reaches the library as it is, which refuses it."""
    from types import SimpleNamespace

    import torch

    from paper_2608_22322_amd import activations as act

    t = SimpleNamespace(dtype=torch.float32, shape=(rows, cols), is_cuda=True, device="cuda", stride=lambda: strides, data_ptr=lambda: A)
    assert act._mat(t, "x", rows, cols, torch.float32) == (A, pitch)
    if rows > 1 and pitch < cols:
        assert _quantize(dtype=0, rows=rows, cols=cols, ld=pitch) == 1


def test_wgrad_refuses_more_weights_than_its_grids_hold():
    need = ctypes.c_size_t(0)
    for out, cols, want in (((1 << 22) - 1, 1 << 17, 4), (1 << 21, (1 << 17) + 1, 4), (1 << 21, 1 << 17, 0), ((1 << 22) - 1, (1 << 29) - 1, 4)):
        assert _status("al_linear_wgrad_workspace_bytes", 1, 64, out, cols, ctypes.byref(need)) == want
