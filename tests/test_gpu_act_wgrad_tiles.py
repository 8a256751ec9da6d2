"""The weight gradient's 128- and 256-wide kernels, unsplit and split, with their joins and bias sums.

Every size is checked against the library's plan, so that a change of the plan's model cannot take a kernel out of the tests. Results are
exact: small integers, whose sums fp32 holds in any order, and 24-bit numbers that meet one token each.
"""
import numpy as np
import pytest
import torch

from tests.act_util import DT, gpu, to_code, wgrad_plan
from tests.test_gpu_act_wgrad import _integers, _run

pytestmark = pytest.mark.gpu

# dtype, tokens, out_features, in_features: tile, splits, bias sums in the product's launch
CASES = [
    ("bf16", 1, 2731, 4200, 128, 1, False), ("bf16", 33, 2731, 4200, 128, 1, False), ("bf16", 161, 2731, 4200, 128, 1, False),
    ("bf16", 225, 2731, 4200, 128, 1, False), ("bf16", 1000, 2100, 4100, 128, 1, False), ("bf16", 2048, 1001, 1750, 128, 4, True),
    ("bf16", 4001, 1100, 1100, 128, 6, True), ("bf16", 4127, 1105, 197, 128, 12, True), ("bf16", 5000, 1001, 2060, 128, 3, True),
    ("bf16", 40000, 512, 512, 128, 32, False), ("bf16", 312, 3563, 4534, 256, 1, False), ("bf16", 340, 3563, 4534, 256, 1, False),
    ("bf16", 3001, 2060, 2055, 256, 3, True), ("bf16", 2555, 4724, 900, 256, 3, True), ("bf16", 8192, 2048, 2048, 256, 4, True),
    ("bf16", 20001, 1100, 700, 256, 16, False),
    ("f32", 1, 2731, 4200, 128, 1, False), ("f32", 33, 2731, 4200, 128, 1, False), ("f32", 97, 2731, 4200, 128, 1, False),
    ("f32", 2048, 1001, 1750, 128, 4, True), ("f32", 4127, 1105, 197, 128, 24, True), ("f32", 20000, 300, 260, 128, 48, False),
    ("f32", 65, 2731, 5700, 256, 1, False), ("f32", 129, 2731, 5700, 256, 1, False), ("f32", 225, 2731, 5700, 256, 1, False),
    ("f32", 2048, 5632, 2048, 256, 1, False), ("f32", 3001, 2060, 2055, 256, 3, True), ("f32", 774, 770, 5157, 256, 3, True),
    ("f32", 40000, 512, 512, 256, 64, False),
]
NAMES = ["-".join(map(str, c[:4])) for c in CASES]


def _planned(dtype, tokens, out, cols, tile, splits, beside):
    got = wgrad_plan(0 if dtype == "f32" else 1, tokens, out, cols)
    assert (got[0], got[1], got[3]) == (tile, splits, beside), "another kernel: choose a size that takes this one"


def _product(dy, x):
    """dy^T x in 64 bits, on the GPU."""
    return torch.mm(dy.double().cuda().t().contiguous(), torch.from_numpy(x).cuda())


@pytest.mark.parametrize("dtype,tokens,out,cols,tile,splits,beside", CASES, ids=NAMES)
def test_integers_are_exact(dtype, tokens, out, cols, tile, splits, beside):
    _planned(dtype, tokens, out, cols, tile, splits, beside)
    for block, pad, shift in ((64, 0, 0), (32, 8, 0), (128, 5, 3)):
        dy, codes, exps, x = _integers(tokens, out, cols, block, tokens + out + block)
        want, total = _product(dy, x), dy.double().sum(0).cuda()
        d, code = gpu(dy.to(DT[dtype]), pad, shift), to_code(codes, exps, cols, block)
        dw, _ = _run(d, code, "f32")
        assert torch.equal(dw.double(), want)
        # scale, shift, base and bias: halves and small integers
        g = torch.Generator().manual_seed(block)
        gamma, beta = (torch.randint(1, 4, (cols,), generator=g) * 0.5).cuda(), torch.randint(-2, 3, (cols,), generator=g).float().cuda()
        base = torch.randint(-9, 10, (out, cols), generator=g).float().cuda()
        full = want * gamma.double() + total[:, None] * beta.double() + base.double()
        assert bool((full.abs() * 8 < 2.0**24).all())  # (so that fp32 holds them)
        dw, db = _run(d, code, "f32", gamma, beta, base, bias=True, in_place=pad == 8)
        assert torch.equal(dw.double(), full) and torch.equal(db.double(), total)
        dw, db = _run(d, code, "bf16", gamma, beta, base.bfloat16(), bias=True)
        assert torch.equal(dw, full.float().bfloat16()) and torch.equal(db, total.float().bfloat16())


def _parts(x):
    """The three bf16 numbers that add up to an fp32 number, each the leading 8 bits of what the ones before it leave."""
    parts = []
    for _ in range(3):
        h = (x.astype(np.float32).view(np.uint32) & 0xFFFF0000).view(np.float32)
        parts.append(h)
        x = x - h
    assert not x.any()
    return parts


def _tokens_met(tokens, out, splits, rng):
    """A token for each output row: the ends of every split and of the whole turns among them, then all in turn or by chance."""
    steps = -(-tokens // 32)
    ends = {0, tokens - 1, tokens // 32 * 32 - 1, tokens // 32 * 32}
    for s in range(splits + 1):
        ends |= {steps * s // splits * 32 + i for i in (-33, -32, -1, 0, 31, 32)}
    ends = [t for t in sorted(ends) if 0 <= t < tokens][:out]
    rest = rng.permutation(max(tokens, out)) % tokens
    return rng.permutation(np.concatenate([ends, rest[: out - len(ends)]]).astype(np.int64))


@pytest.mark.parametrize("dtype,tokens,out,cols,tile,splits,beside", CASES + [
    ("f32", 60, 300, 200, 64, 1, False), ("f32", 100, 300, 200, 64, 2, True), ("f32", 2042, 33, 36, 64, 32, True),
    ("f32", 512, 1024, 1024, 64, 3, True)],
    ids=NAMES + ["f32-60-300-200", "f32-100-300-200", "f32-2042-33-36", "f32-512-1024-1024"])
def test_each_output_from_one_token(dtype, tokens, out, cols, tile, splits, beside):
    """Each column of dy has one number, its product with that token's codes is an output as it is. fp32 numbers have 24 bits, of
    which each of the three parts holds some: one that is lost, doubled or from another turn shows."""
    _planned(dtype, tokens, out, cols, tile, splits, beside)
    rng = np.random.default_rng(tokens + out)
    bits = rng.integers(1 << 7, 1 << 8, out) << 16  # leading 8 bits
    if dtype == "f32":
        bits += (rng.integers(1 << 7, 1 << 8, out) << 8) + rng.integers(0, 1 << 7, out) * 2 + 1
    v = (np.ldexp(bits.astype(np.float64), rng.integers(-30, -10, out)) * rng.choice([-1, 1], out)).astype(np.float32)
    if dtype == "f32":
        assert all(p.all() for p in _parts(v))
    met = _tokens_met(tokens, out, splits, rng)
    dy = np.zeros((tokens, out), np.float32)
    dy[met, np.arange(out)] = v
    nb = -(-cols // 64)
    codes = rng.choice([-1, 1], (tokens, nb * 64)).astype(np.int8)
    codes[:, cols:] = 0
    exps = rng.integers(118, 137, (tokens, nb)).astype(np.uint8)
    sign = torch.from_numpy(codes[:, :cols]).cuda()[torch.from_numpy(met).cuda()].double()
    step = np.ldexp(1.0, exps.astype(int) - 127)
    scale = torch.from_numpy(step).cuda()[torch.from_numpy(met).cuda()].repeat_interleave(64, 1)[:, :cols]
    want = torch.from_numpy(v).cuda().double()[:, None] * sign * scale
    dw, db = _run(gpu(torch.from_numpy(dy).to(DT[dtype]), 3, 1), to_code(codes, exps, cols, 64), "f32", bias=True)
    assert torch.equal(dw.double(), want)
    assert torch.equal(db.cpu(), torch.from_numpy(v))


@pytest.mark.parametrize("dtype,tokens,out,cols,tile,splits,beside", [
    ("bf16", 225, 2731, 4200, 128, 1, False), ("bf16", 2048, 1001, 1750, 128, 4, True), ("bf16", 340, 3563, 4534, 256, 1, False),
    ("bf16", 3001, 2060, 2055, 256, 3, True), ("f32", 97, 2731, 4200, 128, 1, False), ("f32", 2048, 1001, 1750, 128, 4, True),
    ("f32", 129, 2731, 5700, 256, 1, False), ("f32", 3001, 2060, 2055, 256, 3, True)])
def test_values_that_are_no_numbers_stay_in_their_rows_and_columns(dtype, tokens, out, cols, tile, splits, beside):
    """Where tiles overlap too: NaN and infinities of dy stay in their out_feature's row, a code that holds none in its block's columns."""
    _planned(dtype, tokens, out, cols, tile, splits, beside)
    rng = np.random.default_rng(out)
    nb = -(-cols // 64)
    codes = (rng.integers(1, 9, (tokens, nb * 64)) * rng.choice([-1, 1], (tokens, nb * 64))).astype(np.int8)
    codes[:, cols:] = 0
    exps = np.full((tokens, nb), 127, np.uint8)
    rows, blocks = [5, out - tile - 1, out - 1], [1, nb - 1]
    dy = torch.randn(tokens, out, generator=torch.Generator().manual_seed(3))
    dy[tokens - 1, rows[0]], dy[0, rows[1]], dy[tokens // 2, rows[2]] = float("nan"), float("nan"), float("inf")
    for t, b in zip((2, tokens - 1), blocks):
        codes[t, 64 * b:64 * b + 64], exps[t, b] = 0, 255
    dw, _ = _run(gpu(dy.to(DT[dtype])), to_code(codes, exps, cols, 64), "f32")
    bad = torch.zeros(out, cols, dtype=torch.bool, device="cuda")
    bad[rows] = True
    for b in blocks:
        bad[:, 64 * b:64 * b + 64] = True
    assert torch.equal(~torch.isfinite(dw), bad)
    assert bool(torch.isnan(dw[rows[:2]]).all()) and bool(torch.isnan(dw[:, 64:128]).all())
    keep = torch.ones(cols, dtype=torch.bool, device="cuda")
    for b in blocks:
        keep[64 * b:64 * b + 64] = False
    sign = torch.from_numpy(np.sign(codes[tokens // 2, :cols]).astype(np.float32)).cuda()
    assert torch.equal(dw[out - 1][keep], (sign * float("inf"))[keep])


@pytest.mark.parametrize("dtype,tokens,out,cols,tile,splits,beside", [
    ("bf16", 97, 4100, 4200, 128, 1, False), ("f32", 277, 196, 4168, 128, 3, True)])
def test_rows_of_dy_far_apart(dtype, tokens, out, cols, tile, splits, beside):
    """A row pitch of more than 2^25 elements: a 128-wide plan, unsplit and split, taken by the 64-wide kernel in the plan's workspace."""
    _planned(dtype, tokens, out, cols, tile, splits, beside)
    ints, codes, exps, x = _integers(tokens, out, cols, 64, 9)
    ld = (1 << 25) + 8
    dy = torch.empty(tokens * ld, dtype=DT[dtype], device="cuda").view(tokens, ld)[:, 16:16 + out]
    dy.copy_(ints)
    dw, db = _run(dy, to_code(codes, exps, cols, 64), "f32", bias=True)
    assert torch.equal(dw.double(), _product(ints, x)) and torch.equal(db.double(), ints.double().sum(0).cuda())
    beta, base = torch.randint(-2, 3, (cols,)).float().cuda(), torch.randint(-9, 10, (out, cols)).float().cuda()
    dw, _ = _run(dy, to_code(codes, exps, cols, 64), "f32", beta=beta, base=base)
    assert torch.equal(dw.double(), _product(ints, x) + ints.double().sum(0).cuda()[:, None] * beta.double() + base.double())


def test_code_rows_far_apart():
    """Code rows of 2^26 bytes, 2^33 outputs: a 128-wide plan taken by the 64-wide kernel."""
    from paper_2608_22322_amd import activations as act

    tokens, out, cols = 3, 128, 1 << 26
    _planned("bf16", tokens, out, cols, 128, 1, False)
    g = torch.Generator(device="cuda").manual_seed(2)
    codes = torch.randint(-8, 9, (tokens, cols), dtype=torch.int8, device="cuda", generator=g)
    exps = torch.full((tokens, cols // 64), 127, dtype=torch.uint8, device="cuda")
    dy = torch.randint(-4, 5, (tokens, out), device="cuda", generator=g).bfloat16()
    code, dw = act.ActCode(codes, exps, tokens, cols, 64), torch.empty(out, cols, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(act.linear_wgrad_workspace_bytes(dy, code, dw), dtype=torch.uint8, device="cuda")
    act.linear_wgrad(dy, code, dw, ws)
    step = 1 << 22
    for c in range(0, cols, step):
        want = torch.mm(dy.float().t().contiguous(), codes[:, c:c + step].float())  # integers up to 96
        assert torch.equal(dw[:, c:c + step].float(), want), c
