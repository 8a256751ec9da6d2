"""A linear layer's weight gradient from its input's 8-bit code, against 64-bit forms.

The products are exact and summed in fp32, so integers give exact results in any order; for other values a sum of n
products is within n U of the sum of their magnitudes (U = 2^-24), three times as many for fp32 dy.
"""
import numpy as np
import pytest
import torch

from tests.act_util import B16, DT, U, f64, gpu, random_code, to_code

pytestmark = pytest.mark.gpu

# tokens, out_features, in_features: one of each, edges of the tiles, long and short sums, few and many outputs
SIZES = [(1, 1, 1), (1, 40, 33), (2, 130, 70), (31, 128, 128), (32, 129, 127), (33, 257, 96), (64, 256, 256), (65, 250, 300),
         (100, 300, 520), (512, 512, 512), (777, 64, 1001), (1000, 31, 2048), (4096, 136, 72), (6001, 256, 320), (130, 1032, 776),
         (320, 2048, 1280), (192, 1500, 2731)]


def _run(dy, code, grad, gamma=None, beta=None, base=None, bias=False, in_place=False):
    from paper_2608_22322_amd import activations as act

    out, cols = dy.shape[1], code.cols
    dw = torch.full((out, cols), 777.0, dtype=DT[grad], device="cuda")
    if in_place:
        dw.copy_(base)
        base = dw
    db = torch.full((out,), 777.0, dtype=DT[grad], device="cuda") if bias else None
    ws = torch.full((max(256, act.linear_wgrad_workspace_bytes(dy, code, dw)),), 255, dtype=torch.uint8, device="cuda")
    act.linear_wgrad(dy, code, dw, ws, gamma=gamma, beta=beta, base=base, dbias=db)
    return dw, db


def _integers(tokens, out, cols, block, seed):
    """Integers -4..4, codes -8..8 at steps 1/4..2: sums below 2^24 quarters."""
    rng = np.random.default_rng(seed)
    dy = torch.from_numpy(rng.integers(-4, 5, (tokens, out))).float()
    nb = -(-cols // block)
    codes = rng.integers(-8, 9, (tokens, nb * block)).astype(np.int8)
    codes[:, cols:] = 0
    exps = rng.integers(125, 129, (tokens, nb)).astype(np.uint8)
    x = (codes.reshape(tokens, nb, block) * np.ldexp(1.0, exps.astype(int) - 127)[..., None]).reshape(tokens, -1)[:, :cols]
    return dy, codes, exps, x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,out,cols", SIZES)
def test_integers_are_exact(tokens, out, cols, dtype):
    for block, pad, shift in ((64, 0, 0), (32, 8, 0), (128, 5, 3)):
        dy, codes, exps, x = _integers(tokens, out, cols, block, tokens + out)
        want = dy.double().numpy().T @ x
        d = gpu(dy.to(DT[dtype]), pad, shift)
        dw, db = _run(d, to_code(codes, exps, cols, block), "f32", bias=True)
        assert np.array_equal(f64(dw), want)
        assert np.array_equal(f64(db), dy.double().numpy().sum(0))
        base = torch.randint(-9, 10, (out, cols)).float()
        dw, _ = _run(d, to_code(codes, exps, cols, block), "f32", base=base.cuda(), in_place=pad == 8)
        assert np.array_equal(f64(dw), want + base.double().numpy())


@pytest.mark.parametrize("grad", ["bf16", "f32"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,out,cols", SIZES)
def test_values(tokens, out, cols, dtype, grad):
    block = 64
    g = torch.Generator().manual_seed(tokens)
    codes, exps, x = random_code(tokens, cols, block, tokens)
    dy = (1e-2 * torch.randn(tokens, out, generator=g)).to(DT[dtype])
    gamma, beta = 1 + 0.2 * torch.randn(cols, generator=g), 0.2 * torch.randn(cols, generator=g)
    base = (1e-2 * torch.randn(out, cols, generator=g)).to(DT[grad])
    d64, g64, b64, base64 = (t.double().numpy() for t in (dy, gamma, beta, base))
    dw, db = _run(gpu(dy), to_code(codes, exps, cols, block), grad, gamma.cuda(), beta.cuda(), base.cuda(), bias=True)
    n = tokens * (3 if dtype == "f32" else 1)
    prod, size, total = d64.T @ x, np.abs(d64).T @ np.abs(x), d64.sum(0)
    want = prod * g64 + total[:, None] * b64 + base64
    toff = (tokens + 4) * U * np.abs(d64).sum(0)
    tol = (n + 8) * U * (size * np.abs(g64) + np.abs(base64)) + toff[:, None] * np.abs(b64) + 8 * U * np.abs(total[:, None] * b64)
    tol = tol + (B16 * (np.abs(want) + tol) if grad == "bf16" else 0)
    assert (np.abs(f64(dw) - want) <= tol).all()
    assert (np.abs(f64(db) - total) <= toff + (B16 * (np.abs(total) + toff) if grad == "bf16" else 0)).all()


@pytest.mark.parametrize("tokens,out,cols", [(40, 100, 100), (320, 1024, 1024)])
def test_fp32_dy_keeps_its_24_bits(tokens, out, cols):
    """Sums that cancel down to the last bits of dy: only exact products give them."""
    rng = np.random.default_rng(1)
    half = rng.integers(1 << 23, 1 << 24, (tokens // 2, out)).astype(np.float64)
    dy = np.concatenate([half, -(half + rng.integers(1, 4, half.shape))])  # still below 2^24 + 4: 24 bits
    dy = np.clip(dy, -(2.0**24), 2.0**24)
    codes = np.tile(rng.integers(1, 3, (tokens // 2, -(-cols // 64) * 64)).astype(np.int8), (2, 1))
    codes[:, cols:] = 0
    exps = np.full((tokens, -(-cols // 64)), 127, dtype=np.uint8)
    want = dy.T @ codes[:, :cols]
    dw, _ = _run(torch.from_numpy(dy).float().cuda(), to_code(codes, exps, cols, 64), "f32")
    size = np.abs(dy).T @ codes[:, :cols]
    assert (np.abs(f64(dw) - want) <= 3 * tokens * U * size).all()
    one = torch.from_numpy(dy[:1]).float()
    dw, _ = _run(one.cuda(), to_code(codes[:1], exps[:1], cols, 64), "f32")
    assert (np.abs(f64(dw) - one.double().numpy().T @ codes[:1, :cols]) <= 4 * U * np.abs(f64(dw))).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,out,cols", [(70, 90, 200), (192, 512, 512), (200, 520, 584)])
def test_values_that_are_no_numbers_stay_in_their_rows_and_columns(tokens, out, cols, dtype):
    """NaN and infinities of dy reach their out_feature's row, a code that holds none its block's columns, nothing else."""
    codes, exps, x = random_code(tokens, cols, 64, 7)
    codes[:, :cols][codes[:, :cols] == 0] = 1  # no 0 times infinity but where it is meant
    x = np.where(x == 0, 1.0, x)
    dy = torch.randn(tokens, out)
    dy[tokens - 1, 5], dy[3, out - 1] = float("nan"), float("inf")
    codes[2, 64:128], exps[2, 1] = 0, 255
    dw, _ = _run(gpu(dy.to(DT[dtype]), 3, 1), to_code(codes, exps, cols, 64), "f32")
    got = f64(dw)
    bad = np.zeros_like(got, dtype=bool)
    bad[5], bad[out - 1], bad[:, 64:128] = True, True, True
    assert np.isfinite(got[~bad]).all() and not np.isfinite(got[bad]).any()
    assert np.isnan(got[5]).all() and np.isnan(got[:, 64:128]).all()
    inf = np.sign(codes[3, :cols].astype(float)) * np.inf
    keep = np.ones(cols, dtype=bool)
    keep[64:128] = False
    assert np.array_equal(got[out - 1][keep], inf[keep])


def test_no_tokens_and_empty_sides():
    codes = to_code(np.zeros((0, 128), np.int8), np.zeros((0, 2), np.uint8), 100, 64)
    base = torch.randn(50, 100, device="cuda")
    dw, db = _run(torch.empty(0, 50, device="cuda"), codes, "f32", base=base, bias=True)
    assert torch.equal(dw, base) and not db.any()
    dw, _ = _run(torch.empty(0, 50, device="cuda"), codes, "bf16")
    assert not dw.any()
    none = to_code(np.zeros((6, 0), np.int8), np.zeros((6, 0), np.uint8), 0, 64)
    _, db = _run(torch.ones(6, 50, device="cuda"), none, "f32", bias=True)
    assert (db == 6).all()
    _run(torch.ones(6, 0, device="cuda"), to_code(*random_code(6, 100, 64, 1)[:2], 100, 64), "f32")


def test_repeats_on_another_stream_and_in_a_graph():
    """The same bits from call to call, on a side stream and from a replayed graph (with other work between replays)."""
    from paper_2608_22322_amd import activations as act

    codes, exps, _ = random_code(3000, 200, 64, 5)
    c = to_code(codes, exps, 200, 64)
    dy = torch.randn(3000, 120, device="cuda").bfloat16()
    gamma, beta = torch.randn(200, device="cuda"), torch.randn(200, device="cuda")
    first, fb = _run(dy, c, "f32", gamma, beta, bias=True)
    dw, db = torch.empty_like(first), torch.empty_like(fb)
    ws = torch.empty(max(256, act.linear_wgrad_workspace_bytes(dy, c, dw)), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        act.linear_wgrad(dy, c, dw, ws, gamma=gamma, beta=beta, dbias=db)
    s.synchronize()
    assert torch.equal(dw, first) and torch.equal(db, fb)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        act.linear_wgrad(dy, c, dw, ws, gamma=gamma, beta=beta, dbias=db)
    keep = dy.clone()
    for i in range(4):
        dy.copy_(keep * (i + 1))
        dw.fill_(3.0)
        db.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        want, wb = _run(dy, c, "f32", gamma, beta, bias=True)
        assert torch.equal(dw, want) and torch.equal(db, wb)


def test_refusals():
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import activations as act

    c = to_code(*random_code(64, 100, 64, 1)[:2], 100, 64)
    dy, dw = torch.randn(64, 32, device="cuda"), torch.empty(32, 100, device="cuda")
    ws = torch.empty(act.linear_wgrad_workspace_bytes(dy, c, dw), dtype=torch.uint8, device="cuda")
    for call in (lambda: act.linear_wgrad(dy[:63], c, dw, ws), lambda: act.linear_wgrad(dy, c, dw.t(), ws),
                 lambda: act.linear_wgrad(dy, c, dw.half(), ws), lambda: act.linear_wgrad(dy, c, dw, ws, base=dw.bfloat16()),
                 lambda: act.linear_wgrad(dy, c, dw, ws, gamma=torch.ones(99, device="cuda")),
                 lambda: act.linear_wgrad(dy, c, dw, ws, dbias=torch.ones(33, device="cuda")),
                 lambda: act.linear_wgrad(dy, c, torch.empty(100, 32, device="cuda").t(), ws)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(al.ALError) as e:
        act.linear_wgrad(dy, c, dw, ws[:128])
    assert e.value.status == 3
