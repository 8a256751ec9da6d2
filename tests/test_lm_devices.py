"""CPU tests: the operators of a token model run on their operands' GPU or not at all, and check what they are handed."""
from types import SimpleNamespace

import pytest
import torch

from paper_2608_22322_amd import muon, vocab
from tests.test_act_devices import _Lib

A = 1 << 20
SIZE = {torch.float32: 4, torch.bfloat16: 2, torch.int64: 8, torch.int32: 4, torch.uint8: 1}


def _tensor(shape, dtype, dev, strides=None):
    n = 1
    for s in shape:
        n *= s
    at = strides or ((shape[1], 1) if len(shape) == 2 else (1,))
    return SimpleNamespace(dtype=dtype, shape=shape, dim=lambda: len(shape), is_cuda=dev >= 0, device=f"cuda:{dev}", get_device=lambda: dev,
                           stride=lambda i=None: at if i is None else at[i], data_ptr=lambda: A, numel=lambda: n, is_contiguous=lambda: strides is None,
                           element_size=lambda: SIZE[dtype])


T, H, V = 8, 64, 50
F, B = torch.float32, torch.bfloat16
OPERANDS = {"x": ((T, H), F), "y": ((T, H), F), "table": ((V, H), B), "ids": ((T,), torch.int64), "dw": ((V, H), F), "base": ((V, H), F), "h": ((T, H), B), "w": ((V, H), B),
            "dh": ((T, H), B), "loss": ((T,), F), "lse": ((T,), F), "weight": ((T,), F), "ws": ((1 << 20,), torch.uint8)}
CALLS = {
    "orthogonalize": ("x y ws", lambda o, **k: muon.orthogonalize(o["x"], o["y"], o["ws"], **k)),
    "embed_forward": ("table ids x", lambda o, **k: vocab.embed_forward(o["table"], o["ids"], o["x"], **k)),
    "embed_backward": ("x ids dw base ws", lambda o, **k: vocab.embed_backward(o["x"], o["ids"], o["dw"], o["ws"], base=o["base"], **k)),
    "linear_xent": ("h w ids loss lse weight dh dw base ws", lambda o, **k: vocab.linear_xent(
        o["h"], o["w"], o["ids"], o["loss"], o["ws"], weight=o["weight"], lse=o["lse"], dh=o["dh"], dw=o["dw"], base=o["base"], **k)),
}


def _operands(dev, **other):
    o = {k: _tensor(shape, dtype, dev) for k, (shape, dtype) in OPERANDS.items()}
    o.update(other)
    return o


@pytest.fixture
def fake(monkeypatch):
    """A library that only counts, on a machine with two GPUs of which 0 is current."""
    lib = _Lib()
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0)
    for m in (muon, vocab):
        monkeypatch.setattr(m, "lib", lambda: lib)
    return lib


@pytest.mark.parametrize("name", CALLS)
def test_one_gpu(fake, name):
    CALLS[name][1](_operands(0))
    assert fake.calls == ["al_" + name]


@pytest.mark.parametrize("name,odd", [(n, o) for n, (ops, _) in CALLS.items() for o in ops.split()])
def test_an_operand_elsewhere(fake, name, odd):
    shape, dtype = OPERANDS[odd]
    for dev in (1, -1):
        with pytest.raises(ValueError):
            CALLS[name][1](_operands(0, **{odd: _tensor(shape, dtype, dev)}))
    assert fake.calls == []


@pytest.mark.parametrize("name", CALLS)
def test_not_the_current_gpu(fake, name):
    with pytest.raises(ValueError, match="cuda:1"):
        CALLS[name][1](_operands(1))
    with pytest.raises(ValueError, match="cuda:1"):
        CALLS[name][1](_operands(0), stream=SimpleNamespace(cuda_stream=5, device_index=1))
    assert fake.calls == []


BAD = [("embed_forward", "ids", ((T,), torch.int16)), ("embed_forward", "ids", ((T + 1,), torch.int64)), ("embed_forward", "ids", ((T, 1), torch.int64)),
       ("embed_forward", "table", ((V, H + 1), B)), ("embed_backward", "dw", ((V, H + 1), F)), ("embed_backward", "base", ((V, H), B)),
       ("embed_backward", "base", ((V + 1, H), F)), ("embed_backward", "ids", ((T - 1,), torch.int32)), ("linear_xent", "h", ((T, H), F)), ("linear_xent", "w", ((V, H), F)),
       ("linear_xent", "w", ((V, H + 8), B)), ("linear_xent", "loss", ((T + 1,), F)), ("linear_xent", "weight", ((T,), B)), ("linear_xent", "dh", ((T, H + 1), B)),
       ("linear_xent", "dw", ((V, H - 1), F)), ("linear_xent", "base", ((V, H), B)), ("linear_xent", "lse", ((T,), B)), ("orthogonalize", "y", ((T, H + 1), F)),
       ("orthogonalize", "y", ((H, T), F))]


@pytest.mark.parametrize("name,odd,made", BAD)
def test_shapes_and_types(fake, name, odd, made):
    if made[1] not in SIZE:
        SIZE[made[1]] = 2
    with pytest.raises((ValueError, TypeError)):
        CALLS[name][1](_operands(0, **{odd: _tensor(*made, 0)}))
    assert fake.calls == []


@pytest.mark.parametrize("name,odd,strides", [("embed_forward", "ids", (2,)), ("embed_backward", "dw", (H + 8, 1)), ("linear_xent", "dw", (H + 8, 1)),
                                              ("linear_xent", "loss", (2,)), ("linear_xent", "h", (1, T)), ("orthogonalize", "x", (H, 2))])
def test_strides(fake, name, odd, strides):
    with pytest.raises(ValueError):
        CALLS[name][1](_operands(0, **{odd: _tensor(*OPERANDS[odd], 0, strides)}))
    assert fake.calls == []
