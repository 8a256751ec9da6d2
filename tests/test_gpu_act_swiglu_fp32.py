"""The gated activation in fp32, to a few roundings of its 64-bit form at any gate.

Tolerances (U = 2^-24, all relative unless said). e^-gate is within an ulp, 2 U; the sum 1 + e^-gate and the quotient round: sigma within
4 U. Forward: two products more, 6 U. dup: two products, 6 U. dgate = dh up sigma (1 + gate (1 - sigma)): in the factor sigma's error comes in
as |gate| 4 U sigma, 1 - sigma and its product with gate round (2 U |gate| (1 - sigma)), the sum rounds (U); outside it sigma's 4 U
and three products. 5% for the products of such errors; results below the normal numbers round by 2^-149.
"""
import numpy as np
import pytest
import torch

from tests.act_util import U, decode, f64, to_code

pytestmark = pytest.mark.gpu

MORE, LEAST = 1.05, 2.0**-148


def _gates(rows, cols, seed):
    """From -80 to 80 in equal parts, the middle denser (a third within +-3)."""
    rng = np.random.default_rng(seed)
    g = rng.uniform(-80, 80, (rows, cols))
    return np.where(rng.random((rows, cols)) < 1 / 3, rng.uniform(-3, 3, (rows, cols)), g).astype(np.float32)


def _sigma(x):
    return 1 / (1 + np.exp(-x))


@pytest.mark.parametrize("rows,cols", [(3, 100), (64, 1001), (300, 520)])
def test_forward(rows, cols):
    from paper_2608_22322_amd import activations as act

    gate = _gates(rows, cols, cols)
    up = np.random.default_rng(1).normal(size=(rows, cols)).astype(np.float32)
    h = torch.empty(rows, cols, device="cuda")
    act.swiglu_forward(torch.from_numpy(gate).cuda(), torch.from_numpy(up).cuda(), h)
    a, u = gate.astype(np.float64), up.astype(np.float64)
    want = a * _sigma(a) * u
    assert (np.abs(f64(h) - want) <= MORE * 6 * U * np.abs(want) + LEAST).all()


@pytest.mark.parametrize("rows,cols", [(3, 100), (64, 1001), (300, 520)])
def test_backward(rows, cols):
    from paper_2608_22322_amd import activations as act

    rng = np.random.default_rng(cols)
    nb = -(-cols // 32)
    # codes of either sign at steps 2^-6 .. 1/2: gates up to 63
    gc, uc = (rng.integers(-127, 128, (rows, nb * 32)).astype(np.int8) for _ in range(2))
    gc[:, cols:] = uc[:, cols:] = 0
    ge, ue = rng.integers(121, 127, (rows, nb)).astype(np.uint8), np.full((rows, nb), 121, np.uint8)
    a, u = decode(gc, ge, cols, 32), decode(uc, ue, cols, 32)
    dh = rng.normal(size=(rows, cols)).astype(np.float32)
    dgate, dup = torch.empty(rows, cols, device="cuda"), torch.empty(rows, cols, device="cuda")
    act.swiglu_backward(torch.from_numpy(dh).cuda(), to_code(gc, ge, cols, 32), to_code(uc, ue, cols, 32), dgate, dup)
    d, p, rest = dh.astype(np.float64), _sigma(a), _sigma(-a)
    want = d * a * p
    assert (np.abs(f64(dup) - want) <= MORE * 6 * U * np.abs(want) + LEAST).all()
    factor = 1 + a * rest
    want = d * u * p * factor
    inner = np.abs(a) * (4 * p + 2 * rest) + np.abs(factor)
    off = np.abs(d * u * p) * U * (np.abs(factor) * 7 + inner)
    assert (np.abs(f64(dgate) - want) <= MORE * off + LEAST).all()


def test_gates_past_the_exponential():
    """Where e^-gate overflows sigma is 0; where it vanishes sigma is 1; no number stays none."""
    from paper_2608_22322_amd import activations as act

    gate = torch.tensor([[-3e38, -200.0, -90.0, 0.0, 200.0, 3e38, float("nan"), float("inf")]])
    h = torch.empty(1, 8, device="cuda")
    act.swiglu_forward(gate.cuda(), torch.ones(1, 8, device="cuda"), h)
    got = h.cpu()[0]
    assert got[:2].abs().max() == 0 and abs(float(got[2])) < 2.0**-120 and got[3] == 0
    assert got[4] == 200.0 and got[5] == torch.tensor(3e38) and bool(got[6].isnan()) and got[7] == float("inf")
