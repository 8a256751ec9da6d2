"""Orthogonalised matrices and momentum steps in one 11-bit part (and in two) against bounds that a wrong result cannot meet: 5% of the result at most, 15%
for a few rows.

Large matrices: errors of thousands of independent roundings, compared with those of the same roundings in another order of sums (`rounded`), which agree to a few per cent; half as much again is
allowed for one part, three times for two parts (where the fp32 sums matter as much and are formed otherwise). Small ones: a bound from the singular values that they have."""
import numpy as np
import pytest
import torch

from tests.act_util import DT, f64, gpu, out_like, untouched
from tests.ortho_util import COEFS, newton_schulz, rounded

pytestmark = pytest.mark.gpu

OUT = {"f32": 2.0**-24, "bf16": 2.0**-8}
ROOM = {1: 1.5, 2: 3.0}


def matrix(rows, cols, dtype, seed):
    x = np.random.default_rng(seed).normal(size=(rows, cols)) * 1e-3
    return torch.from_numpy(x.astype(np.float32)).to(DT[dtype])


def run(x, view, parts):
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import muon

    ws = al.workspace(muon.orthogonalize_workspace_bytes(x, view, parts))
    ws.fill_(0xff)
    muon.orthogonalize(x, view, ws, parts=parts)
    torch.cuda.synchronize()


def defined(wide, eps=1e-7):
    """The 64-bit definition on the GPU, rows <= cols."""
    a, b, c = COEFS
    y = wide.double() / (wide.double().norm() + eps)
    for _ in range(5):
        q = y @ y.t().contiguous()
        y = a * y + (b * q + c * (q @ q)) @ y
    return y


def allowed(wide, y, parts):
    """Relative Frobenius norm."""
    return ROOM[parts] * max(float((rounded(wide, parts, pairs).double() - y).norm() / y.norm()) for pairs in (False, True))


@pytest.mark.parametrize("rows,cols", [(500, 64), (64, 301), (129, 60), (301, 63), (1001, 130), (131, 1750), (100, 4100), (4100, 100), (300, 701), (701, 301), (1536, 4200), (4200, 1536), (2500, 640),
                                       (2048, 2048)])
@pytest.mark.parametrize("dtype,out,parts", [("bf16", "bf16", None), ("bf16", "bf16", 2), ("f32", "bf16", 1), ("bf16", "f32", 1), ("bf16", "f32", 2)])
def test_types_and_pitches(rows, cols, dtype, out, parts):
    x = matrix(rows, cols, dtype, rows * 7 + cols)
    held = gpu(x, pad=5, shift=3)
    view, buf = out_like(rows, cols, DT[out], pad=3, shift=1)
    run(held, view, parts)
    wide = held.float() if rows <= cols else held.float().t().contiguous()
    y = defined(wide)
    off = float(((view if rows <= cols else view.t()).double() - y).norm() / y.norm())
    p = parts or 1
    tol = allowed(wide, y, p) + OUT[out]
    print(f"{rows} x {cols} {dtype} -> {out}, {p} parts: off {off:.2e} of {tol:.2e}", flush=True)
    assert tol < (0.05 if p == 1 else 0.005)
    assert off <= tol
    assert untouched(view, buf)


def spectral_bound(seen, parts, out_unit, exact_start):
    """Frobenius norm of the error allowed to the last X. In the singular vectors of X a step maps an error's symmetric part by divided differences of f(t) = a t + b t^3 + c t^5, which are values of
    f' between the smallest and the largest singular value, and the rest by (f(s) + f(t)) / (s + t) and f(s) / s: at most the largest f(s) / s. The other terms are those of `tolerance`: what is held
    in 11 or 21 bits (u), fp32 sums (s), F: Frobenius norm, S: spectral norm."""
    a, b, c = COEFS
    u = 2.0**-11 if parts == 1 else 2.0**-21
    f = lambda m: float(np.sqrt((m * m).sum()))  # noqa: E731
    e = 0.0 if exact_start else u * f(seen[0])
    for i, x in enumerate(seen[:-1]):
        wide = x if x.shape[0] <= x.shape[1] else x.T
        sv = np.linalg.svd(wide, compute_uv=False)
        t = np.linspace(sv.min() * 0.99, sv.max() * 1.01, 2001)
        ell = max(np.abs(a + 3 * b * t**2 + 5 * c * t**4).max(), np.abs(a + b * t**2 + c * t**4).max())
        s = (max(wide.shape) / 32 + 5) * 2.0**-24
        gram = wide @ wide.T
        poly = b * gram + c * gram @ gram
        top = sv.max()
        e = ell * (e + (u * f(x) if i > 0 else 0.0))
        e += (u * f(gram) + s * f(x) ** 2) * (abs(b) + 2 * abs(c) * top**2) * top
        e += (u * f(poly) + abs(c) * s * f(gram) ** 2) * top + s * f(poly) * f(x) + 2 * 2.0**-24 * f(seen[i + 1])
    return 1.1 * e + out_unit * f(seen[-1])


SMALL = [(1, 1), (1, 2), (1, 300), (300, 1), (1, 4097), (2, 65), (65, 2), (3, 1000), (1000, 3), (5, 5000), (5000, 5)]


@pytest.mark.parametrize("rows,cols", SMALL)
@pytest.mark.parametrize("dtype,out,parts", [("bf16", "bf16", 1), ("f32", "f32", 1), ("bf16", "f32", 2)])
def test_a_few_rows(rows, cols, dtype, out, parts):
    x = matrix(rows, cols, dtype, rows * 7 + cols)
    held = gpu(x, pad=5, shift=3)
    view, buf = out_like(rows, cols, DT[out], pad=3, shift=1)
    run(held, view, parts)
    want, seen = newton_schulz(f64(x))
    off, tol = np.sqrt(((f64(view) - want) ** 2).sum()), spectral_bound(seen, parts, OUT[out], dtype == "bf16")
    print(f"{rows} x {cols} {dtype} -> {out}, {parts} parts: off {off:.2e} of {tol:.2e}", flush=True)
    assert tol < 0.15 * np.sqrt((want**2).sum())
    assert off <= tol
    assert untouched(view, buf)


@pytest.mark.parametrize("uf8", [True, False])
@pytest.mark.parametrize("grad_bf16", [True, False])
@pytest.mark.parametrize("parts", [1, 2])
@pytest.mark.parametrize("shapes", [[(500, 64), (64, 301), (700, 301), (129, 60)], [(500, 60), (64, 301)], [(2048, 2048), (2048, 5632), (300, 701), (500, 64)]])
def test_the_parameters_of_a_momentum_step(uf8, grad_bf16, parts, shapes):
    """What a step leaves in the parameters beside their decay, with a momentum from before: its error a share of the update, and the parameters' own rounding."""
    import paper_2608_22322_amd as al

    g = torch.Generator(device="cuda").manual_seed(31)
    spec = al.Spec(al.UF8 if uf8 else al.FP32, 256)
    sts, before, old = [], [], []
    for r, c in shapes:
        m, meta = al.alloc_state(r * c, spec)
        start = torch.empty(r * c, device="cuda").normal_(0, 5e-4, generator=g)
        if uf8:
            al.quantize(al.UF8, start, 256, 0.0, m, meta)
            al.dequantize(al.UF8, m, meta, r * c, 256, start)
        else:
            m.copy_(start)
        grad = torch.empty(r, c, device="cuda").normal_(0, 1e-3, generator=g)
        sts.append(al.ParamState(torch.empty(r, c, device="cuda").normal_(0, 0.02, generator=g), grad.bfloat16() if grad_bf16 else grad, r, c, m=m, m_meta=meta))
        before.append(sts[-1].param.double())
        old.append(start.view(r, c).double())
    cfg = al.muon_cfg(lr=2e-2, weight_decay=0.1, parts=parts, grad_bf16=grad_bf16, m=spec)
    al.muon_step(sts, cfg, 1, al.workspace(al.muon_workspace_bytes(sts, cfg)))
    for st, p, m in zip(sts, before, old):
        g = st.grad.double()
        m = (cfg.beta * m + (1.0 - cfg.beta) * g).float().double()
        u = (cfg.beta * m + (1.0 - cfg.beta) * g).float()
        wide = u if st.rows <= st.cols else u.t().contiguous()
        y = defined(wide)
        size = cfg.lr * 0.2 * max(st.rows, st.cols) ** 0.5
        want = p * (1.0 - cfg.lr * cfg.weight_decay) - size * (y if st.rows <= st.cols else y.t())
        off, share = float((st.param.double() - want).norm()), allowed(wide, y, parts)
        tol = share * size * float(y.norm()) + 2.0**-24 * float(want.norm())
        print(f"{st.rows} x {st.cols}, {parts} parts: off {off:.2e} of {tol:.2e}", flush=True)
        assert share < (0.05 if parts == 1 else 0.005)
        assert off <= tol
