"""Cross entropy of a linear head whose weight holds minus infinities."""
import numpy as np
import pytest
import torch

from tests.act_util import U, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,hidden,vocab", [(3, 72, 90), (1, 8, 5), (300, 200, 777), (600, 136, 5000), (2048, 328, 8192)])
@pytest.mark.parametrize("grad", [False, True])
def test_a_weight_of_minus_infinity(tokens, hidden, vocab, grad):
    """A feature that is minus infinity for some columns and positive in every token takes them out of the softmax, wherever it stands: also among the last features of a head whose features are
    a multiple of 8 and not of 64. dh has no value (probability zero times infinity), the loss and dw do."""
    from paper_2608_22322_amd import vocab as voc
    import paper_2608_22322_amd as al

    rng = np.random.default_rng(vocab)
    for column in (hidden - 1, 0, hidden - 8):
        h = torch.from_numpy(rng.normal(size=(tokens, hidden))).bfloat16()
        w = torch.from_numpy(rng.normal(size=(vocab, hidden)) / hidden**0.5).bfloat16()
        h[:, column] = h[:, column].abs() + 0.5
        out = rng.random(vocab) < 0.3
        out[0], out[-1] = False, True
        w[torch.from_numpy(out), column] = float("-inf")
        target = torch.from_numpy(rng.choice(np.flatnonzero(~out), tokens))
        x, y = f64(h), f64(w)
        z = x @ np.where(np.isinf(y), 0.0, y).T
        span = (hidden / 32 + 6) * U * (np.abs(x) @ np.abs(np.where(np.isinf(y), 0.0, y)).T).max(1)
        z[:, out] = -np.inf
        top = z.max(1, keepdims=True)
        lse = np.log(np.exp(z - top).sum(1, keepdims=True)) + top
        want = lse[:, 0] - z[np.arange(tokens), target.numpy()]
        dw = torch.empty(w.shape, device="cuda") if grad else None
        loss, held, weight = torch.empty(tokens, device="cuda"), h.cuda(), w.cuda()
        voc.linear_xent(held, weight, target.cuda(), loss, al.workspace(voc.linear_xent_workspace_bytes(held, weight, None, dw)), dw=dw)
        off = np.abs(f64(loss) - want)
        # twice the logits' error (of lse, of the target's), the exponentials' and the sums' as for exact logits
        assert (off <= 2 * span + U * (2 * 20 + 44) + 4 * U * np.abs(want)).all(), column
        if grad:
            d = np.exp(z - lse)
            d[np.arange(tokens), target.numpy()] -= 1.0
            got = f64(dw)
            assert not got[out].any()
            bound = (np.abs(d) * (2.0**-16 + 2 * span[:, None] + U * 100)).T @ np.abs(x) + U * (tokens / 32 + 14) * (np.abs(d).T @ np.abs(x)) + U * np.abs(d.T @ x)
            # (the target's d = p - 1 is off by p's error)
            p = np.exp(z - lse)
            bound += (p * (2 * span[:, None] + U * 100)).T @ np.abs(x)
            assert (np.abs(got - d.T @ x) <= bound + 1e-30).all(), column
