"""The weight gradient at the ends of its promised sizes: whole grids, every output written."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("out,cols", [((1 << 22) - 1, 8), ((1 << 22) - 1, 70), (8, (1 << 29) - 1)])
def test_longest_sides(out, cols):
    from paper_2608_22322_amd import activations as act

    tokens, block = 3, 64
    nb = -(-cols // block)
    g = torch.Generator(device="cuda").manual_seed(1)
    codes = torch.randint(-8, 9, (tokens, nb * block), dtype=torch.int8, device="cuda", generator=g)
    codes[:, cols:] = 0
    code = act.ActCode(codes, torch.full((tokens, nb), 127, dtype=torch.uint8, device="cuda"), tokens, cols, block)
    dy = torch.randint(-4, 5, (tokens, out), device="cuda", generator=g).bfloat16()
    dw, db = torch.full((out, cols), 777.0, dtype=torch.bfloat16, device="cuda"), torch.full((out,), 777.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(act.linear_wgrad_workspace_bytes(dy, code, dw), dtype=torch.uint8, device="cuda")
    act.linear_wgrad(dy, code, dw, ws, dbias=db)
    assert torch.equal(db.float(), dy.float().sum(0))
    step = 1 << 22
    for n in range(0, out, step):
        for c in range(0, cols, step):
            # three products, integers up to 96
            want = sum(dy[t, n:n + step].float()[:, None] * codes[t, c:min(c + step, cols)].float() for t in range(tokens))
            assert torch.equal(dw[n:n + step, c:c + step].float(), want), (n, c)
