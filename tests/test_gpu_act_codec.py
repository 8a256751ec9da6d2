"""The activation code E8 on the GPU: codes and exponents are equal to the definition's, decoding is exact."""
import numpy as np
import pytest
import torch

from tests.act_util import DT, decode, encode, f64, gpu, out_like, untouched

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (1, 7), (3, 8), (2, 31), (5, 32), (3, 33), (4, 63), (3, 129), (7, 500), (2, 1001), (257, 96), (33, 4096)]


def _values(rows, cols, dtype, seed):
    """Values over many magnitudes, with zeros, zero rows, ties and denormals."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(rows, cols)) * np.exp2(rng.integers(-20, 20, (rows, 1 + (cols - 1) // 16)).repeat(16, 1)[:, :cols])
    x[rng.random((rows, cols)) < 0.05] = 0.0
    if rows > 2:
        x[1] = 0.0
        x[2] = np.ldexp(rng.integers(-255, 256, cols) * 0.5, rng.integers(-148, -120))  # exact halves, denormal steps
    return torch.from_numpy(x).to(torch.float32).to(DT[dtype])


def _save(x, block):
    from paper_2608_22322_amd import activations as act

    c = act.alloc_code(*x.shape, block)
    act.quantize(x, c)
    return c


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("block", [32, 64, 128])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_codes_are_the_definitions(rows, cols, block, dtype):
    from paper_2608_22322_amd import activations as act

    x = _values(rows, cols, dtype, rows * 1000 + cols)
    want_c, want_e = encode(x.double().numpy(), block)
    for pad, shift in ((0, 0), (5, 0), (8, 3)):
        c = _save(gpu(x, pad, shift), block)
        assert np.array_equal(c.exps.cpu().numpy(), want_e)
        assert np.array_equal(c.codes.cpu().numpy(), want_c)
        values = decode(want_c, want_e, cols, block)
        for out_dtype in ("f32", "bf16"):
            out, buf = out_like(rows, cols, DT[out_dtype], pad, shift)
            act.dequantize(c, out)
            assert np.array_equal(f64(out), values) and untouched(out, buf)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_blocks_with_infinities_and_nan_decode_to_nan(dtype):
    from paper_2608_22322_amd import activations as act

    x = torch.randn(4, 200, dtype=torch.float32)
    x[0, 3], x[1, 64], x[2, 199], x[3, 130] = float("inf"), float("-inf"), float("nan"), float("nan")
    x = x.to(DT[dtype])
    c = _save(x.cuda(), 64)
    want_c, want_e = encode(x.double().numpy(), 64)
    assert np.array_equal(c.exps.cpu().numpy(), want_e) and int((c.exps == 255).sum()) == 4
    out = torch.empty(4, 200, device="cuda")
    act.dequantize(c, out)
    assert np.array_equal(f64(out), decode(want_c, want_e, 200, 64), equal_nan=True)


def test_largest_and_smallest_magnitudes():
    from paper_2608_22322_amd import activations as act

    top = np.finfo(np.float32).max
    x = torch.tensor([[top, -top, 1.0, 0.0] * 8, [2.0**-126, -(2.0**-149), 2.0**-130, 0.0] * 8, [1e-45] * 32, [-0.0] * 32])
    c = _save(x.cuda(), 32)
    want_c, want_e = encode(x.double().numpy(), 32)
    assert np.array_equal(c.exps.cpu().numpy(), want_e) and np.array_equal(c.codes.cpu().numpy(), want_c)
    out = torch.empty(4, 32, device="cuda")
    act.dequantize(c, out)
    assert np.array_equal(f64(out), decode(want_c, want_e, 32, 32)) and bool(torch.isfinite(out).all())


def test_empty_matrices_and_another_stream():
    from paper_2608_22322_amd import activations as act

    for rows, cols in ((0, 64), (4, 0)):
        c = act.alloc_code(rows, cols, 64)
        x = torch.empty(rows, cols, device="cuda")
        act.quantize(x, c)
        act.dequantize(c, x)
    x = torch.randn(64, 1000)
    s = torch.cuda.Stream()
    xd, c, out = x.cuda(), act.alloc_code(64, 1000, 128), torch.empty(64, 1000, device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    act.quantize(xd, c, stream=s)
    act.dequantize(c, out, stream=s)
    s.synchronize()
    assert np.array_equal(f64(out), decode(*encode(x.numpy(), 128), 1000, 128))


def test_refusals():
    from paper_2608_22322_amd import activations as act

    x = torch.randn(8, 100, device="cuda")
    c = act.alloc_code(8, 100, 64)
    for bad in (x[:4], x[:, :99], x.t(), x.half(), x.cpu(), x[0], x[:, ::2]):
        with pytest.raises(ValueError):
            act.quantize(bad, c)
        with pytest.raises(ValueError):
            act.dequantize(c, bad)
    with pytest.raises(ValueError):
        act.ActCode(c.codes, c.exps, 8, 100, 48)
    with pytest.raises(ValueError):
        act.ActCode(c.codes, c.exps, 9, 100, 64)
    with pytest.raises(ValueError):
        act.ActCode(c.codes.cpu(), c.exps, 8, 100, 64)


def test_expanded_rows_are_refused():
    """Views whose rows overlap hold fewer elements than rows x cols."""
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import activations as act

    c = act.alloc_code(8, 100, 64)
    wide = torch.randn(1, 100, device="cuda")
    full = torch.randn(8, 100, device="cuda")
    for bad in (wide.expand(8, 100), torch.randn(200, device="cuda").as_strided((8, 100), (1, 1))):
        with pytest.raises(al.ALError):
            act.quantize(bad, c)
        with pytest.raises(al.ALError):
            act.dequantize(c, bad)
        with pytest.raises(al.ALError):
            act.norm_forward(act.RMS, bad, torch.empty_like(full))
        with pytest.raises(al.ALError):
            act.norm_backward(act.RMS, bad, c, None, torch.ones(8, device="cuda"), torch.empty_like(full))
        with pytest.raises(al.ALError):
            act.swiglu_forward(full, bad, torch.empty_like(full))
        with pytest.raises(al.ALError):
            act.linear_wgrad(bad, c, torch.empty(100, 100, device="cuda"), al.workspace(1 << 22))
    c1 = act.alloc_code(1, 100, 64)
    act.quantize(wide.expand(1, 100), c1)  # a single row has no pitch
