"""Cross entropy of logits that are known exactly: confident tokens and large logits, whose loss and gradients must not pay for the logits' own size."""
import numpy as np
import pytest
import torch

from tests.act_util import U, f64

pytestmark = pytest.mark.gpu

MARKED = 16  # classes that a column of their own lifts by the margin


def known(tokens, vocab, offset, margin, seed):
    """bf16 (h, w), targets and logits in binary64: offset + a multiple of 2^-4 within 2, lifted by `margin` for the target. A logit is the sum of three bf16 numbers (the offset's and the
    noise's bits in pieces of 8) and the margin, all multiples of 2^-4 below 2^13: exact in fp32 in any order. The last column of w is 1 where h has 0."""
    rng = np.random.default_rng(seed)
    z = offset + rng.integers(-32, 33, vocab) / 16.0
    w = np.zeros((vocab, 64))
    rest = z.copy()
    for k in range(3):
        w[:, k] = torch.from_numpy(rest).to(torch.bfloat16).double().numpy()
        rest -= w[:, k]
    assert not rest.any()
    w[np.arange(MARKED), 4 + np.arange(MARKED)] = margin
    w[:, 63] = 1.0
    h = np.zeros((tokens, 64))
    h[:, :3] = 1.0
    target = np.arange(tokens) % MARKED
    h[np.arange(tokens), 4 + target] = 1.0
    return torch.from_numpy(h).bfloat16(), torch.from_numpy(w).bfloat16(), torch.from_numpy(target), h @ w.T


def call(h, w, target, grad=None, scale=1.0):
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import vocab as voc

    h, w = h.cuda(), w.cuda()
    loss, lse = torch.empty(len(target), device="cuda"), torch.empty(len(target), device="cuda")
    dh = dw = None
    if grad:
        dh, dw = torch.empty(h.shape, device="cuda", dtype=grad), torch.empty(w.shape, device="cuda", dtype=grad)
    ws = al.workspace(voc.linear_xent_workspace_bytes(h, w, dh, dw))
    ws.fill_(0xff)
    voc.linear_xent(h, w, target.cuda(), loss, ws, scale=scale, lse=lse, dh=dh, dw=dw)
    torch.cuda.synchronize()
    return loss, lse, dh, dw


@pytest.mark.parametrize("offset", [0.0, 30.0, 100.0, 3000.0])
@pytest.mark.parametrize("margin", [4.0, 8.0, 12.0])
def test_confident_tokens(offset, margin):
    """loss = log(1 + r), r the sum of exp(z - z[target]) over the other columns. Differences of logits are exact. An exp is off by 2^-24 (2 |x| + 4) of itself (its argument times log2(e),
    the hardware's two units); a sum that holds the 1 is rounded by 2^-24 at most (half a step below 2) in each of 16 additions of a lane, 2 of its row, 8 and 6 of the row's groups; the logarithm
    turns the sum's error into as much of its own and is off by 2 units of its result."""
    h, w, target, z = known(200, 1000, offset, margin, int(offset + margin))
    loss, lse, _, _ = call(h, w, target)
    x = z - z[np.arange(200), target.numpy()][:, None]
    e = np.exp(x)
    e[np.arange(200), target.numpy()] = 0.0
    r = e.sum(1)
    want = np.log1p(r)
    tol = U * (e * (2 * np.abs(x) + 4)).sum(1) + 32 * U + 4 * U * want
    off = np.abs(f64(loss) - want)
    print(f"offset {offset}, margin {margin}: off {off.max():.2e} of {tol.min():.2e}, {(off / want).max():.2e} of the loss", flush=True)
    assert (off <= tol).all()
    top = z[np.arange(200), target.numpy()]
    assert (np.abs(f64(lse) - (top + want)) <= tol + U * np.abs(top + want)).all()


@pytest.mark.parametrize("offset", [0.0, 100.0, 3000.0])
@pytest.mark.parametrize("tokens,vocab", [(200, 1000), (2100, 2000)])
def test_a_row_of_d_sums_to_nothing(offset, tokens, vocab):
    """The probabilities of a row sum to 1, so a row of d (held in 16 bits for an fp32 gradient: off by 2^-16 of each element) sums to 0: what the column of ones in w makes of it in dh.
    A probability is off by 2^-24 (2 |x| + 8) with x = log p, and by the sum's error, 2^-24 (2 |x| + 4) in the mean and 40 additions' 2^-24; the product's sum by 2^-24 (vocab / 32 + 12)."""
    h, w, target, z = known(tokens, vocab, offset, 5.0, 3)
    _, _, dh, dw = call(h, w, target, torch.float32)
    top = z.max(1, keepdims=True)
    p = np.exp(z - top)
    p /= p.sum(1, keepdims=True)
    d = p.copy()
    d[np.arange(tokens), target.numpy()] -= 1.0
    lost = U * (2 * np.abs(np.log(p)) + 8)
    off_d = 2.0**-16 * np.abs(d) + p * (lost + (p * lost).sum(1, keepdims=True) + 40 * U) + U * np.abs(d)
    size = np.abs(d).sum(1)
    tol = off_d.sum(1) + U * (vocab / 32 + 12) * size
    off = np.abs(f64(dh)[:, 63])
    print(f"offset {offset}: off {off.max():.2e} of {tol.min():.2e}", flush=True)
    assert (off <= tol).all()
    want, bound = d.T @ f64(h), off_d.T @ f64(h) + U * (tokens / 32 + 14) * (np.abs(d).T @ f64(h))
    assert (np.abs(f64(dw) - want) <= bound + 1e-30).all()
