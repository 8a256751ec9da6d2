"""Layer and RMS norm and their backward pass against 64-bit forms.

Tolerances. A row's fp32 sum of n terms goes through at most D = 40 additions of one chain (8 in a chunk's tree, up to 8
chunks, 6 across lanes, 16 across wavefronts), so a mean of terms t is off by at most D U mean|t|, with U = 2^-24. The
statistics are therefore off by D U mean|x| (mean) and, relative, (D / 2 + 8) U (rstd); the rest are a few
roundings of the terms themselves. A bf16 result adds 2^-8 of itself.
"""
import numpy as np
import pytest
import torch

from tests.act_util import B16, DT, U, decode, f64, gpu, out_like, random_code, to_code, untouched

pytestmark = pytest.mark.gpu

D = 40
COLS = [1, 7, 8, 40, 64, 65, 500, 512, 513, 1001, 1024, 1750, 2048, 2056, 4096, 4097, 5632, 8192, 8200, 11008, 16384, 16385, 20001]


def _inputs(rows, cols, dtype, seed, offset=0.3):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, cols, generator=g) * torch.exp(0.5 * torch.randn(cols, generator=g)) + offset).to(DT[dtype])
    gamma = 1 + 0.2 * torch.randn(cols, generator=g)
    beta = 0.2 * torch.randn(cols, generator=g)
    return x, gamma, beta


def _stats(x, layer, eps):
    mu = x.mean(1, keepdims=True) if layer else np.zeros((x.shape[0], 1))
    return mu, 1 / np.sqrt(((x - mu) ** 2).mean(1, keepdims=True) + eps)


def _forward(kind, layer, x, gamma, beta, eps, code=None, pad=0, shift=0):
    from paper_2608_22322_amd import activations as act

    rows, cols = x.shape
    y, buf = out_like(rows, cols, x.dtype, pad, shift)
    mean = torch.empty(rows, device="cuda") if layer else None
    rstd = torch.empty(rows, device="cuda")
    act.norm_forward(kind, gpu(x, pad, shift), y, mean, rstd, gamma=None if gamma is None else gamma.cuda(),
                     beta=None if beta is None else beta.cuda(), eps=eps, code=code)
    assert untouched(y, buf)
    return y, mean, rstd


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", COLS)
def test_forward(cols, dtype, kind):
    from paper_2608_22322_amd import activations as act

    layer, eps = kind == "layer", 1e-5
    for rows, block, pad, shift in ((1, 64, 0, 0), (5, 128, 3, 1), (18, 32, 8, 0)):
        x, gamma, beta = _inputs(rows, cols, dtype, cols + rows)
        beta = beta if layer else None
        code = act.alloc_code(rows, cols, block) if rows != 5 else None
        y, mean, rstd = _forward(act.LAYER if layer else act.RMS, layer, x, gamma, beta, eps, code, pad, shift)
        x64 = x.double().numpy()
        mu, r = _stats(x64, layer, eps)
        dmu = D * U * np.abs(x64).mean(1, keepdims=True) if layer else 0 * mu
        # rstd: the deviations are off by dmu (a bias they all share) and the square, the mean and the root round
        dr = r * ((D / 2 + 8) * U + (r * dmu) ** 2 + r * dmu * 2 * U)
        assert (np.abs(f64(rstd)[:, None] - r) <= dr).all()
        if layer:
            assert (np.abs(f64(mean)[:, None] - mu) <= dmu + U * np.abs(mu)).all()
        xh = (x64 - mu) * r
        dxh = r * dmu + np.abs(x64 - mu) * dr + 4 * U * np.abs(xh)
        want = xh * gamma.numpy() + (beta.numpy() if layer else 0)
        tol = dxh * np.abs(gamma.numpy()) + 4 * U * (np.abs(want) + (np.abs(beta.numpy()) if layer else 0))
        tol = tol + (B16 * (np.abs(want) + tol) if dtype == "bf16" else 0)
        assert (np.abs(f64(y) - want) <= tol).all()
        if code is not None:
            _check_code(code, xh, dxh, cols, block)


def _check_code(code, want, off, cols, block):
    """The code of values that are `want` to within `off`: its steps are those of the largest magnitude, its values are
    the nearest ones (one step where the code is at its end)."""
    codes, exps = code.codes.cpu().numpy(), code.exps.cpu().numpy()
    nb = exps.shape[1]
    pad = ((0, 0), (0, nb * block - cols))
    top = np.pad(np.abs(want), pad).reshape(-1, nb, block).max(-1)
    slack = np.pad(off, pad).reshape(-1, nb, block).max(-1)

    def exp_of(a):
        return np.where(a > 0, np.maximum(np.frexp(a)[1] + 120, 1), 1)

    assert (exps >= exp_of(np.maximum(top - slack, 0))).all() and (exps <= exp_of(top + slack)).all()
    step = np.ldexp(1.0, exps.astype(int) - 127).repeat(block, 1)[:, :cols]
    ends = np.abs(codes[:, :cols].astype(int)) == 127
    assert (np.abs(decode(codes, exps, cols, block) - want) <= np.where(ends, 1.0, 0.5) * step + off).all()
    assert not codes[:, cols:].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_variants(dtype):
    """No weight, in place, a row without variance, a row that holds a NaN or an infinity, a large common offset."""
    from paper_2608_22322_amd import activations as act

    x, _, _ = _inputs(6, 777, dtype, 5)
    x[1] = 0.0
    x[2] = 3.0
    x[3, 5] = float("nan")
    x[4, 700] = float("inf")
    for kind, layer in ((act.LAYER, True), (act.RMS, False)):
        code = act.alloc_code(6, 777, 64)
        d = x.cuda()
        act.norm_forward(kind, d, d, eps=1e-6, code=code)
        got = f64(d)
        assert np.isnan(got[3]).all() and np.isnan(got[4, 700]) and (code.exps[3] == 255).all()
        assert not got[1].any() and not code.codes[1].any()
        x64 = x.double().numpy()
        mu, r = _stats(x64, layer, 1e-6)
        want = (x64 - mu) * r
        # row 2 has no deviation but its mean's rounding (exact here up to D U |x|), times r = 1e3
        tol = np.abs(want) * ((D + 16) * U + (B16 if dtype == "bf16" else 0)) + r * D * U * np.abs(x64).mean(1, keepdims=True)
        for i in (0, 2, 5):
            assert (np.abs(got[i] - want[i]) <= tol[i] * (1 + B16)).all(), i
        y = torch.empty_like(d)
        act.norm_forward(kind, x.cuda(), y, eps=1e-6)
        assert torch.equal(y.nan_to_num(9.0), d.nan_to_num(9.0))
    x, _, _ = _inputs(4, 4096, "f32", 6, offset=1000.0)
    y, mean, rstd = _forward(act.LAYER, True, x, None, None, 1e-5)
    x64 = x.double().numpy()
    mu, r = _stats(x64, True, 1e-5)
    dmu = D * U * np.abs(x64).mean(1, keepdims=True)
    assert (np.abs(f64(y) - (x64 - mu) * r) <= r * dmu + np.abs(x64 - mu) * r * ((D + 16) * U + (r * dmu) ** 2)).all()


def _backward_reference(dy, xh, r, gamma, add, layer):
    a = dy * gamma
    v = a - xh * (a * xh).mean(1, keepdims=True) - (a.mean(1, keepdims=True) if layer else 0)
    dx = v * r + add
    size = (np.abs(a) + np.abs(xh) * np.abs(a * xh).mean(1, keepdims=True) + (np.abs(a).mean(1, keepdims=True) if layer else 0)) * r
    return dx, size, (dy * xh).sum(0), dy.sum(0)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("source", ["x", "code"])
@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("cols", COLS)
def test_backward(cols, dtype, grad, source, kind):
    from paper_2608_22322_amd import activations as act

    layer = kind == "layer"
    k = act.LAYER if layer else act.RMS
    for rows, block, pad, shift, add in ((1, 64, 0, 0, False), (6, 128, 3, 1, True), (37 if cols < 9000 else 9, 32, 8, 0, True)):
        x, gamma, _ = _inputs(rows, cols, dtype, cols + rows)
        g = torch.Generator().manual_seed(cols)
        dy = (1e-2 * torch.randn(rows, cols, generator=g)).to(DT[dtype])
        dy[rows // 2] = 0.0
        res = (1e-2 * torch.randn(rows, cols, generator=g)).to(DT[dtype]) if add else None
        mu, r = _stats(x.double().numpy(), layer, 1e-5)
        mean, rstd = torch.from_numpy(mu[:, 0]).float(), torch.from_numpy(r[:, 0]).float()
        mu, r = mean.double().numpy()[:, None], rstd.double().numpy()[:, None]
        if source == "code":
            codes, exps, xh = random_code(rows, cols, block, cols)
            src, dxh = to_code(codes, exps, cols, block), 0.0
        else:
            src = gpu(x, pad, shift)
            xh = (x.double().numpy() - mu) * r
            dxh = 2 * U * np.abs(xh)
        dx, buf = out_like(rows, cols, DT[dtype], pad, shift)
        dg = torch.empty(cols, dtype=DT[grad], device="cuda")
        db = torch.empty(cols, dtype=DT[grad], device="cuda") if layer else None
        ws = torch.empty(max(256, act.norm_backward_workspace_bytes(k, rows, cols, DT[dtype])), dtype=torch.uint8, device="cuda")
        act.norm_backward(k, gpu(dy, pad, shift), src, mean.cuda() if layer else None, rstd.cuda(), dx, gamma=gamma.cuda(),
                          dgamma=dg, dbeta=db, add=None if res is None else gpu(res, pad, shift), ws=ws)
        assert untouched(dx, buf)
        dy64, a64 = dy.double().numpy(), 0 if res is None else res.double().numpy()
        want, size, wg, wb = _backward_reference(dy64, xh, r, gamma.double().numpy(), a64, layer)
        tol = size * (D + 16) * U + 2 * U * np.abs(a64) + 2 * U * np.abs(want)
        tol = tol + (B16 * (np.abs(want) + tol) if dtype == "bf16" else 0)
        assert (np.abs(f64(dx) - want) <= tol).all()
        # sums over the rows: at most `rows` additions in a chain
        for got, w, s in ((dg, wg, (np.abs(dy64) * (np.abs(xh) + dxh)).sum(0)), (db, wb, np.abs(dy64).sum(0))):
            if got is None:
                continue
            t = (rows + 4) * U * s
            t = t + (B16 * (np.abs(w) + t) if grad == "bf16" else 0)
            assert (np.abs(f64(got) - w) <= t).all()


@pytest.mark.parametrize("rows", [0, 1, 2, 5, 64, 300, 1500, 5000])
@pytest.mark.parametrize("cols", [96, 1300, 2500])
def test_weight_gradients_over_many_rows(rows, cols):
    """Integers: every sum is exact, whatever its order, so a lost or doubled row shows."""
    from paper_2608_22322_amd import activations as act

    g = torch.Generator().manual_seed(rows)
    dy = torch.randint(-3, 4, (rows, cols), generator=g).float()
    x = torch.randint(-3, 4, (rows, cols), generator=g).float()
    one, zero = torch.ones(rows, device="cuda"), torch.zeros(rows, device="cuda")
    dg, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(max(256, act.norm_backward_workspace_bytes(act.LAYER, rows, cols, torch.float32)), dtype=torch.uint8, device="cuda")
    act.norm_backward(act.LAYER, dy.cuda(), x.cuda(), zero, one, torch.empty(rows, cols, device="cuda"), dgamma=dg, dbeta=db, ws=ws)
    assert torch.equal(dg.cpu(), (dy * x).sum(0)) and torch.equal(db.cpu(), dy.sum(0))
    only = torch.empty(cols, device="cuda")
    act.norm_backward(act.LAYER, dy.cuda(), x.cuda(), zero, one, torch.empty(rows, cols, device="cuda"), dbeta=only, ws=ws)
    assert torch.equal(only, db)
    act.norm_backward(act.LAYER, dy.cuda(), x.cuda(), zero, one, torch.empty(rows, cols, device="cuda"))


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_backward_against_differences(kind):
    """Central differences of the 64-bit forward pass (error about h^2 = 1e-8 of the third derivative)."""
    from paper_2608_22322_amd import activations as act

    layer, rows, cols, h = kind == "layer", 3, 21, 1e-4
    k = act.LAYER if layer else act.RMS
    x, gamma, beta = _inputs(rows, cols, "f32", 11)
    w = torch.randn(rows, cols, generator=torch.Generator().manual_seed(1))
    x64, g64, b64, w64 = (t.double().numpy() for t in (x, gamma, beta, w))

    def loss(x, g, b):
        mu, r = _stats(x, layer, 1e-5)
        return (w64 * ((x - mu) * r * g + (b if layer else 0))).sum()

    def slope(f, v):
        out = np.zeros_like(v)
        for i in np.ndindex(v.shape):
            p, m = v.copy(), v.copy()
            p[i] += h
            m[i] -= h
            out[i] = (f(p) - f(m)) / (2 * h)
        return out

    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    act.norm_forward(k, x.cuda(), torch.empty(rows, cols, device="cuda"), mean if layer else None, rstd, eps=1e-5)
    dx, dg = torch.empty(rows, cols, device="cuda"), torch.empty(cols, device="cuda")
    db = torch.empty(cols, device="cuda") if layer else None
    ws = torch.empty(max(256, act.norm_backward_workspace_bytes(k, rows, cols, torch.float32)), dtype=torch.uint8, device="cuda")
    act.norm_backward(k, w.cuda(), x.cuda(), mean if layer else None, rstd, dx, gamma=gamma.cuda(), dgamma=dg, dbeta=db, ws=ws)
    assert np.abs(f64(dx) - slope(lambda v: loss(v, g64, b64), x64)).max() < 2e-5
    assert np.abs(f64(dg) - slope(lambda v: loss(x64, v, b64), g64)).max() < 2e-5
    if layer:
        assert np.abs(f64(db) - slope(lambda v: loss(x64, g64, v), b64)).max() < 2e-5


def test_residual_gradient_in_place_and_repeats():
    """add may be dx itself; two calls give the same bits."""
    from paper_2608_22322_amd import activations as act

    rows, cols = 300, 2050
    x, gamma, _ = _inputs(rows, cols, "bf16", 3)
    dy, add = torch.randn(rows, cols).bfloat16().cuda(), torch.randn(rows, cols).bfloat16().cuda()
    rstd, xd, gd = torch.rand(rows, device="cuda"), x.cuda(), gamma.cuda()
    ws = torch.empty(act.norm_backward_workspace_bytes(act.RMS, rows, cols), dtype=torch.uint8, device="cuda")
    res = []
    for _ in range(2):
        dx, dg = add.clone(), torch.empty(cols, device="cuda")
        act.norm_backward(act.RMS, dy, xd, None, rstd, dx, gamma=gd, dgamma=dg, add=dx, ws=ws)
        res.append((dx, dg))
    apart = torch.empty_like(dy)
    act.norm_backward(act.RMS, dy, xd, None, rstd, apart, gamma=gd, add=add)
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1]) and torch.equal(res[0][0], apart)


def test_refusals():
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import activations as act

    x, y = torch.randn(8, 100, device="cuda"), torch.empty(8, 100, device="cuda")
    v, r = torch.ones(100, device="cuda"), torch.ones(8, device="cuda")
    with pytest.raises(ValueError):
        act.norm_forward(act.RMS, x, y[:7], rstd=r)
    with pytest.raises(ValueError):
        act.norm_forward(act.RMS, x, y.bfloat16(), rstd=r)
    with pytest.raises(ValueError):
        act.norm_forward(act.RMS, x, y, rstd=r, gamma=v[:99])
    with pytest.raises(ValueError):
        act.norm_forward(act.RMS, x, y, rstd=r, code=act.alloc_code(8, 99, 64))
    for bad in (dict(kind=act.RMS, beta=v), dict(kind=act.RMS, mean=r), dict(kind=7), dict(kind=act.RMS, eps=-1.0)):
        kind = bad.pop("kind")
        with pytest.raises(al.ALError):
            act.norm_forward(kind, x, y, **bad)
    dg = torch.empty(100, device="cuda")
    with pytest.raises(al.ALError) as e:  # weight gradients need the workspace
        act.norm_backward(act.RMS, x, x, None, r, y, dgamma=dg)
    assert e.value.status == 3
    with pytest.raises(al.ALError):  # a layer norm from x needs its mean
        act.norm_backward(act.LAYER, x, y, None, r, torch.empty_like(x))
    with pytest.raises(al.ALError):  # in place over dy
        act.norm_backward(act.RMS, x, y, None, r, x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [513, 1025, 4097, 12289, 16385, 16901, 24577])
def test_in_place_where_a_row_ends_in_another_wavefront(cols, dtype):
    """The chunk that a row ends in belongs to another wavefront than the one before it: y over x, dx over add."""
    from paper_2608_22322_amd import activations as act

    rows = 33
    x, gamma, _ = _inputs(rows, cols, dtype, cols)
    d, apart, rstd, gd = x.cuda(), torch.empty(rows, cols, dtype=DT[dtype], device="cuda"), torch.empty(rows, device="cuda"), gamma.cuda()
    act.norm_forward(act.RMS, d, apart, rstd=rstd, gamma=gd)
    dy, add = torch.randn(rows, cols).to(DT[dtype]).cuda(), torch.randn(rows, cols).to(DT[dtype]).cuda()
    want = torch.empty_like(add)
    act.norm_backward(act.RMS, dy, d, None, rstd, want, gamma=gd, add=add)
    for _ in range(5):
        over = add.clone()
        act.norm_backward(act.RMS, dy, d, None, rstd, over, gamma=gd, add=over)
        assert torch.equal(over, want)
        y = d.clone()
        act.norm_forward(act.RMS, y, y, gamma=gd)
        assert torch.equal(y, apart)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("cols", [100, 20000])
def test_no_rows_give_zero_weight_gradients_without_a_workspace(cols, kind):
    from paper_2608_22322_amd import activations as act

    k = act.LAYER if kind == "layer" else act.RMS
    assert act.norm_backward_workspace_bytes(k, 0, cols, torch.float32) == 0
    none, rows = torch.empty(0, cols, device="cuda"), torch.empty(0, device="cuda")
    dg = torch.full((cols,), 7.0, device="cuda")
    db = torch.full((cols,), 7.0, device="cuda") if kind == "layer" else None
    act.norm_backward(k, none, none, rows if kind == "layer" else None, rows, torch.empty(0, cols, device="cuda"), dgamma=dg, dbeta=db)
    assert not dg.any() and (db is None or not db.any())
