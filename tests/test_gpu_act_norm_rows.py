"""Norm forward at row counts on both sides of the rule that takes a wavefront or a workgroup for a row."""
import numpy as np
import pytest
import torch

from tests.act_util import B16, U, f64
from tests.test_gpu_act_norm import D, _check_code, _forward, _inputs, _stats

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("cols", [1025, 1100, 2041, 2048])
@pytest.mark.parametrize("rows", [2047, 2048, 2051])
def test_forward(rows, cols, kind):
    """Tolerances as at few rows (tests/test_gpu_act_norm.py): the chains of a sum are no longer here."""
    from paper_2608_22322_amd import activations as act

    layer, eps, block = kind == "layer", 1e-5, 64
    x, gamma, beta = _inputs(rows, cols, "bf16", cols)
    code = act.alloc_code(rows, cols, block)
    y, mean, rstd = _forward(act.LAYER if layer else act.RMS, layer, x, gamma, beta if layer else None, eps, code, 3, 1)
    x64 = x.double().numpy()
    mu, r = _stats(x64, layer, eps)
    dmu = D * U * np.abs(x64).mean(1, keepdims=True) if layer else 0 * mu
    dr = r * ((D / 2 + 8) * U + (r * dmu) ** 2 + r * dmu * 2 * U)
    assert (np.abs(f64(rstd)[:, None] - r) <= dr).all()
    if layer:
        assert (np.abs(f64(mean)[:, None] - mu) <= dmu + U * np.abs(mu)).all()
    xh = (x64 - mu) * r
    dxh = r * dmu + np.abs(x64 - mu) * dr + 4 * U * np.abs(xh)
    want = xh * gamma.numpy() + (beta.numpy() if layer else 0)
    tol = dxh * np.abs(gamma.numpy()) + 4 * U * (np.abs(want) + (np.abs(beta.numpy()) if layer else 0))
    assert (np.abs(f64(y) - want) <= tol + B16 * (np.abs(want) + tol)).all()
    _check_code(code, xh, dxh, cols, block)
    # in place, the same bits
    d = x.cuda()
    act.norm_forward(act.LAYER if layer else act.RMS, d, d, gamma=gamma.cuda(), beta=beta.cuda() if layer else None, eps=eps)
    assert torch.equal(d, y)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [64, 1025, 1100, 1536, 2048, 4096])
def test_a_row_gives_the_same_bits_among_many_rows_and_few(cols, dtype, kind):
    from paper_2608_22322_amd import activations as act

    rows, few, layer = 2100, 33, kind == "layer"
    x, gamma, beta = _inputs(rows, cols, dtype, cols)
    res = []
    for d in (x.cuda(), x[:few].cuda()):
        n = d.shape[0]
        y, mean, rstd, code = torch.empty_like(d), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), act.alloc_code(n, cols)
        act.norm_forward(act.LAYER if layer else act.RMS, d, y, mean if layer else None, rstd, gamma=gamma.cuda(),
                         beta=beta.cuda() if layer else None, code=code)
        res.append((y[:few], mean[:few], rstd[:few], code.codes[:few], code.exps[:few]))
    assert all(torch.equal(p, q) for p, q in zip(*res))
