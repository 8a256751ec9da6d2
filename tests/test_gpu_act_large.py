"""Matrices whose offsets do not fit 32 bits, rows far apart, and every operator in a replayed graph."""
import numpy as np
import pytest
import torch

from tests.act_util import f64, random_code, to_code

pytestmark = pytest.mark.gpu


def test_offsets_past_32_bits():
    """2.2e9 elements, the last rows alone not zero: what is read and written there is right, in codes and in sums."""
    from paper_2608_22322_amd import activations as act

    rows, cols, last = 208_000, 10_560, 40
    assert rows * cols > 1 << 31
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(last, cols).bfloat16()
    x[-last:] = tail.cuda()
    code, small = act.alloc_code(rows, cols, 64), act.alloc_code(last, cols, 64)
    act.quantize(x, code)
    act.quantize(tail.cuda(), small)
    assert torch.equal(code.codes[-last:], small.codes) and torch.equal(code.exps[-last:], small.exps)
    assert not code.codes[:last].any()
    dy = torch.zeros(rows, 32, dtype=torch.bfloat16, device="cuda")
    dy[-last:] = torch.randn(last, 32).bfloat16().cuda()
    dw, want = torch.empty(32, cols, device="cuda"), torch.empty(32, cols, device="cuda")
    ws = torch.empty(act.linear_wgrad_workspace_bytes(dy, code, dw), dtype=torch.uint8, device="cuda")
    act.linear_wgrad(dy, code, dw, ws)
    act.linear_wgrad(dy[-last:], small, want, ws)
    # (the same products, added in another order: 40 of them, the others 0)
    size = dy[-last:].float().abs().t() @ tail.cuda().float().abs() * 1.02
    assert bool(((dw - want).abs() <= 2 * 42 * 2.0**-24 * size).all())
    rstd, y = torch.empty(rows, device="cuda"), torch.empty_like(x)
    act.norm_forward(act.RMS, x, y, rstd=rstd)
    ref = torch.empty(last, cols, dtype=torch.bfloat16, device="cuda")
    act.norm_forward(act.RMS, tail.cuda(), ref)
    assert torch.equal(y[-last:], ref) and not y[:last].any()
    act.dequantize(code, y)
    act.dequantize(small, ref)
    assert torch.equal(y[-last:], ref)


@pytest.mark.parametrize("tokens,out,cols", [(5, 300, 400), (70, 130, 140)])
def test_rows_of_dy_far_apart(tokens, out, cols):
    """A row pitch of more than 2^25 elements."""
    from paper_2608_22322_amd import activations as act

    ld = (1 << 25) + 8
    buf = torch.empty(tokens * ld, dtype=torch.bfloat16, device="cuda")
    dy = buf.view(tokens, ld)[:, 16:16 + out]
    dy.copy_(torch.randint(-4, 5, (tokens, out)))
    codes, exps, x = random_code(tokens, cols, 64, 3)
    codes, exps = np.clip(codes, -8, 8), np.full_like(exps, 127)
    dw = torch.empty(out, cols, device="cuda")
    code = to_code(codes, exps, cols, 64)
    ws = torch.empty(max(256, act.linear_wgrad_workspace_bytes(dy, code, dw)), dtype=torch.uint8, device="cuda")
    act.linear_wgrad(dy, code, dw, ws)
    assert np.array_equal(f64(dw), f64(dy).T @ codes[:, :cols].astype(np.float64))


def test_every_operator_in_a_replayed_graph():
    """Captured once, replayed with new inputs and other work between: every replay is the eager result."""
    from paper_2608_22322_amd import activations as act

    rows, cols = 700, 520
    x, dy = torch.randn(rows, cols, device="cuda").bfloat16(), torch.randn(rows, cols, device="cuda").bfloat16()
    gamma = torch.randn(cols, device="cuda")

    def buffers():
        return dict(y=torch.empty_like(x), mean=torch.empty(rows, device="cuda"), rstd=torch.empty(rows, device="cuda"), dx=torch.empty_like(x),
                    dg=torch.empty(cols, device="cuda"), db=torch.empty(cols, device="cuda"), h=torch.empty_like(x), a=torch.empty_like(x),
                    b=torch.empty_like(x), out=torch.empty_like(x), codes=[act.alloc_code(rows, cols, 64) for _ in range(4)],
                    dw=torch.empty(cols, cols, device="cuda"))

    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")

    def run(s):
        c = s["codes"]
        act.norm_forward(act.LAYER, x, s["y"], s["mean"], s["rstd"], gamma=gamma, beta=gamma, code=c[0])
        act.swiglu_forward(s["y"], x, s["h"], c[1], c[2])
        act.swiglu_backward(dy, c[1], c[2], s["a"], s["b"], h_code=c[3])
        act.linear_wgrad(s["a"], c[0], s["dw"], ws, gamma=gamma, beta=gamma)
        act.norm_backward(act.LAYER, s["b"], c[0], None, s["rstd"], s["dx"], gamma=gamma, dgamma=s["dg"], dbeta=s["db"], add=dy, ws=ws)
        act.dequantize(c[3], s["out"])

    s, eager = buffers(), buffers()
    assert act.linear_wgrad_workspace_bytes(s["a"], s["codes"][0], s["dw"]) <= ws.numel()
    run(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(s)
    for i in range(4):
        x.copy_(torch.randn(rows, cols, device="cuda") * (i + 1))
        g.replay()
        torch.cuda.synchronize()
        run(eager)
        torch.cuda.synchronize()
        for k, v in s.items():
            if k != "codes":
                assert torch.equal(v, eager[k]), (i, k)
