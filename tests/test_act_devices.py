"""CPU tests: the activation operators run on their operands' GPU or not at all."""
import contextlib
from types import SimpleNamespace

import pytest
import torch

from paper_2608_22322_amd import activations as act

A = 1 << 20


class _Lib:
    """Takes the place of the library: notes the calls that reach it."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append(name) or 0


def _tensor(rows, cols, dtype, dev):
    shape = (rows, cols) if cols else (rows,)
    n = rows * (cols or 1)
    return SimpleNamespace(dtype=dtype, shape=shape, dim=lambda: len(shape), is_cuda=dev >= 0, device=f"cuda:{dev}", get_device=lambda: dev,
                           stride=lambda: (cols, 1), data_ptr=lambda: A, numel=lambda: n, is_contiguous=lambda: True,
                           element_size=lambda: {torch.float32: 4, torch.uint8: 1, torch.int8: 1}[dtype])


ROWS, COLS = 8, 128
CALLS = {  # operands, and the call with them
    "quantize": ("x code.codes code.exps", lambda o, **k: act.quantize(o["x"], o["code"], **k)),
    "dequantize": ("x code.codes code.exps", lambda o, **k: act.dequantize(o["code"], o["x"], **k)),
    "norm_forward": ("x y mean rstd gamma beta code.codes code.exps", lambda o, **k: act.norm_forward(
        act.LAYER, o["x"], o["y"], o["mean"], o["rstd"], gamma=o["gamma"], beta=o["beta"], code=o["code"], **k)),
    "norm_backward": ("x y mean rstd z gamma dgamma dbeta add ws", lambda o, **k: act.norm_backward(
        act.LAYER, o["x"], o["y"], o["mean"], o["rstd"], o["z"], gamma=o["gamma"], dgamma=o["dgamma"], dbeta=o["dbeta"], add=o["add"],
        ws=o["ws"], **k)),
    "norm_backward from the code": ("x rstd z code.codes code.exps", lambda o, **k: act.norm_backward(
        act.RMS, o["x"], o["code"], None, o["rstd"], o["z"], **k)),
    "swiglu_forward": ("x y z code.codes code.exps code2.codes code2.exps", lambda o, **k: act.swiglu_forward(
        o["x"], o["y"], o["z"], o["code"], o["code2"], **k)),
    "swiglu_backward": ("x y z code.codes code.exps code2.codes code2.exps code3.codes code3.exps", lambda o, **k: act.swiglu_backward(
        o["x"], o["code"], o["code2"], o["y"], o["z"], h_code=o["code3"], **k)),
    "linear_wgrad": ("x code.codes code.exps dw ws gamma beta base dbias", lambda o, **k: act.linear_wgrad(
        o["x"], o["code"], o["dw"], o["ws"], gamma=o["gamma"], beta=o["beta"], base=o["base"], dbias=o["dbias"], **k)),
}


def _operands(dev, odd=None, other=None):
    """All on GPU `dev`, the one called `odd` on `other`."""

    def at(name):
        return other if name == odd else dev

    f = torch.float32
    o = {k: _tensor(ROWS, COLS, f, at(k)) for k in ("x", "y", "z", "add")}
    o.update({k: _tensor(ROWS, 0, f, at(k)) for k in ("mean", "rstd")})
    o.update({k: _tensor(COLS, 0, f, at(k)) for k in ("gamma", "beta", "dgamma", "dbeta", "dbias")})
    o.update({k: _tensor(COLS, COLS, f, at(k)) for k in ("dw", "base")})
    o["ws"] = _tensor(1 << 20, 0, torch.uint8, at("ws"))
    for k in ("code", "code2", "code3"):
        o[k] = act.ActCode(_tensor(ROWS, COLS, torch.int8, at(k + ".codes")), _tensor(ROWS, COLS // 64, torch.uint8, at(k + ".exps")), ROWS, COLS, 64)
    return o


@pytest.fixture
def library(monkeypatch):
    """A library that only counts, on a machine with two GPUs of which 0 is current."""
    lib = _Lib()
    monkeypatch.setattr(act, "lib", lambda: lib)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0)
    return lib


@pytest.mark.parametrize("name", CALLS)
def test_operands_of_the_current_gpu(library, name):
    CALLS[name][1](_operands(0))
    CALLS[name][1](_operands(0), stream=SimpleNamespace(cuda_stream=5, device_index=0))
    assert len(library.calls) == 2


@pytest.mark.parametrize("name", CALLS)
def test_operands_of_another_gpu_are_refused(library, name):
    """The null stream's handle is that of the current GPU: the kernel would run there, on another GPU's pointers."""
    with pytest.raises(ValueError, match="cuda:1"):
        CALLS[name][1](_operands(1))
    with pytest.raises(ValueError, match="cuda:1"):
        CALLS[name][1](_operands(0), stream=SimpleNamespace(cuda_stream=5, device_index=1))
    assert not library.calls


@pytest.mark.parametrize("name,odd", [(n, k) for n in CALLS for k in CALLS[n][0].split()])
def test_operands_of_two_gpus_are_refused(library, name, odd):
    for other in (1, -1):  # -1: host memory
        if other < 0 and "." in odd:
            continue  # (ActCode itself refuses it)
        with pytest.raises(ValueError):
            CALLS[name][1](_operands(0, odd, other))
    assert not library.calls


def test_a_block_runs_on_its_own_gpu(monkeypatch):
    """Each pass of the MLP block makes the block's GPU the current one."""
    from paper_2608_22322_amd import mlp

    inside, seen = [], []

    @contextlib.contextmanager
    def device(d):
        inside.append(d)
        yield
        inside.pop()

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(mlp, "adamw_step", lambda *a, **k: seen.append(list(inside)))
    monkeypatch.setattr(act, "norm_forward", lambda *a, **k: seen.append(list(inside)))
    monkeypatch.setattr(act, "swiglu_forward", lambda *a, **k: None)
    monkeypatch.setattr(act, "swiglu_backward", lambda *a, **k: seen.append(list(inside)))
    monkeypatch.setattr(act, "linear_wgrad", lambda *a, **k: None)
    monkeypatch.setattr(act, "norm_backward", lambda *a, **k: None)
    net = object.__new__(mlp.SwigluMLP)
    net.device, net.eps, net.states, net.cfg, net.step_ws, net.arr = "cuda:1", 1e-5, [], None, None, None
    t, h, f = 3, 4, 5
    net.param = {"gate": torch.zeros(f, h), "up": torch.zeros(f, h), "down": torch.zeros(h, f), "norm": torch.ones(1, h)}
    net.weight = {k: net.param[k].clone() for k in ("gate", "up", "down")}
    net.grad = {k: torch.zeros_like(v) for k, v in net.param.items()}
    net.n, net.a, net.b, net.h = torch.zeros(t, h), torch.zeros(t, f), torch.zeros(t, f), torch.zeros(t, f)
    net.rstd = net.xhat = net.gate_code = net.up_code = net.h_code = net.ws = None
    net.forward(torch.zeros(t, h))
    net.backward(torch.zeros(t, h))
    net.step(1)
    assert seen == [["cuda:1"]] * 3 and not inside
