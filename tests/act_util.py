"""Plain 64-bit forms of the 8-bit activation operators, on the CPU, for the tests."""
import numpy as np
import torch

U = 2.0**-24  # unit roundoff of fp32
B16 = 2.0**-8  # of bf16 (8 significant bits)
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def gpu(t, pad=0, shift=0):
    """A GPU copy of a matrix as a slice of a wider buffer: `pad` more columns, the slice from column `shift`."""
    rows, cols = t.shape
    buf = torch.full((rows, cols + pad + shift), float("nan") if t.is_floating_point() else 0, dtype=t.dtype, device="cuda")
    view = buf[:, shift:shift + cols]
    view.copy_(t)
    return view


def out_like(rows, cols, dtype, pad=0, shift=0):
    """(output slice, its whole buffer): the buffer is filled with a value that a kernel must leave alone outside it."""
    buf = torch.full((rows, cols + pad + shift), 777.0, dtype=dtype, device="cuda")
    return buf[:, shift:shift + cols], buf


def untouched(view, buf):
    """Whether the buffer still holds the fill value outside the slice."""
    seen = buf.clone()
    shift = (view.data_ptr() - buf.data_ptr()) // buf.element_size()
    seen[:, shift:shift + view.shape[1]] = 777.0
    return bool((seen == 777.0).all())


def encode(x, block):
    """E8 codes by definition: (int8 [rows, nb * block], uint8 [rows, nb]), from any array of fp32 numbers."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    nb = -(-cols // block)
    v = np.zeros((rows, nb * block))
    v[:, :cols] = x
    v = v.reshape(rows, nb, block)
    bad = ~np.isfinite(v).all(-1)
    v = np.where(bad[..., None], 0.0, v)
    a = np.abs(v).max(-1)
    _, k = np.frexp(a)  # a = f 2^k, f in [1/2, 1): floor(log2 a) = k - 1
    e = np.where(a > 0, np.maximum(k - 1 + 121, 1), 1)
    codes = np.clip(np.rint(np.ldexp(v, (127 - e)[..., None])), -127, 127)
    codes[bad] = 0
    e[bad] = 255
    return codes.astype(np.int8).reshape(rows, nb * block), e.astype(np.uint8)


def decode(codes, exps, cols, block):
    rows, nb = exps.shape
    v = codes.reshape(rows, nb, block).astype(np.float64)
    s = np.ldexp(1.0, exps.astype(np.int64) - 127)[..., None]
    v = np.where(exps[..., None] == 255, np.nan, v * s)
    return v.reshape(rows, nb * block)[:, :cols]


def random_code(rows, cols, block, seed, sigma=1.0):
    """(codes, exps, values) of normal values, as numpy arrays."""
    rng = np.random.default_rng(seed)
    codes, exps = encode(rng.normal(0.0, sigma, (rows, cols)).astype(np.float32), block)
    return codes, exps, decode(codes, exps, cols, block)


def to_code(codes, exps, cols, block):
    from paper_2608_22322_amd import activations as act

    return act.ActCode(torch.from_numpy(codes).cuda(), torch.from_numpy(exps).cuda(), codes.shape[0], cols, block)


def f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def wgrad_plan(dtype, tokens, out, cols):
    """(tile, splits, slabs, beside) that the library takes for a weight gradient; dtype: 0 fp32, 1 bf16."""
    import ctypes

    import paper_2608_22322_amd as al

    plan = (ctypes.c_int32 * 4)()
    al.check(al.lib().al_diag_wgrad_plan(dtype, tokens, out, cols, plan))
    return plan[0], plan[1], plan[2], bool(plan[3])
