"""Matrices past 32-bit offsets, and the time that the largest of them take."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _best(f, times=3):
    """ms of the fastest of some runs."""
    f()
    best = float("inf")
    for _ in range(times):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


def test_a_long_matrix_steps_in_the_time_of_its_products():
    """One product step of 2^21 x 512: besides what al_orthogonalize reads and writes (x twice, X0 and X once each way, the result: 20 bytes an element) the momentum step moves the gradient, the
    momentum, the update twice and the parameters: 24 more. The same products: no more than three times as long."""
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import lib, muon
    import ctypes

    rows, cols = 1 << 21, 512
    g = torch.empty(rows, cols, device="cuda", dtype=torch.bfloat16).normal_()
    m, meta = al.alloc_state(rows * cols, al.Spec(al.UF8, 256))
    st = [al.ParamState(torch.zeros(rows, cols, device="cuda"), g, rows, cols, m=m, m_meta=meta)]
    cfg = al.muon_cfg(parts=1, steps=1)
    ws = al.workspace(al.muon_workspace_bytes(st, cfg))
    step = _best(lambda: al.muon_step(st, cfg, 1, ws))
    x = g.float()
    need = ctypes.c_size_t(0)
    al.check(lib().al_orthogonalize_workspace_bytes(rows, cols, ctypes.byref(al.ortho_cfg(steps=1, parts=1)), ctypes.byref(need)))
    assert need.value <= ws.numel()
    alone = _best(lambda: muon.orthogonalize(x, x, ws, steps=1, parts=1))
    print(f"momentum step {step:.2f} ms, the products {alone:.2f} ms", flush=True)
    assert step < 3 * alone


LONG, SHORT = 1 << 21, 2056  # 2^32 elements and 2^24 more


def _parts_of(n, size=1 << 17):
    return [slice(i, min(n, i + size)) for i in range(0, n, size)]


def _orthogonal(g, picked):
    """Some rows (tall) or columns (wide) of the 64-bit definition of 5 steps: every X is X0 times a polynomial of X0's gram matrix, or that times X0."""
    a, b, c = 3.4445, -4.7750, 2.0315
    tall = g.shape[0] > g.shape[1]
    gram = torch.zeros(SHORT, SHORT, dtype=torch.float64, device="cuda")
    for p in _parts_of(LONG):
        x = (g[p] if tall else g[:, p].t()).double().contiguous()
        gram += x.t().contiguous() @ x
    norm = gram.trace().sqrt() + 1e-7
    gram /= norm * norm
    eye = torch.eye(SHORT, dtype=torch.float64, device="cuda")
    all_ = eye / norm
    for _ in range(5):
        m = a * eye + b * gram + c * (gram @ gram)
        all_, gram = all_ @ m, m @ gram @ m
    return [((g[p] if tall else g[:, p].t()).double() @ all_) for p in picked]


# the first rows, the ones that hold elements 2^31 and 2^32, the last ones
PICKED = [slice(0, 100), slice((1 << 31) // SHORT - 50, (1 << 31) // SHORT + 50), slice((1 << 32) // SHORT - 50, (1 << 32) // SHORT + 50), slice(LONG - 100, LONG)]


@pytest.mark.parametrize("tall", [True, False])
def test_orthogonalised_past_32_bits(tall):
    """One part leaves a few 1e-3 of a matrix whose singular values are nearly equal; an offset that lost bits would read or write other rows, and leave errors of the order of the result: 5%."""
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import muon

    x = torch.empty((LONG, SHORT) if tall else (SHORT, LONG), device="cuda", dtype=torch.bfloat16).normal_()
    out = torch.full_like(x, float("nan"))
    muon.orthogonalize(x, out, al.workspace(muon.orthogonalize_workspace_bytes(x, out)))
    for p, want in zip(PICKED, _orthogonal(x, PICKED)):
        got = (out[p] if tall else out[:, p].t()).double()
        off = float((got - want).norm() / want.norm())
        print(f"from {p.start}: off {off:.1e}", flush=True)
        assert off < 0.05
    assert all(bool((out[p] if tall else out[:, p]).isfinite().all()) for p in _parts_of(LONG))


def test_a_momentum_step_past_32_bits():
    """From a zero momentum the update is the gradient times a number. Codes of the blocks at the end: the nearest to 127 m / absmax, m = 0.05 g rounded once."""
    import paper_2608_22322_amd as al

    g = torch.empty(LONG, SHORT, device="cuda", dtype=torch.bfloat16).normal_()
    n = LONG * SHORT
    m, meta = al.alloc_state(n, al.Spec(al.UF8, 256))
    st = [al.ParamState(torch.zeros(LONG, SHORT, device="cuda"), g, LONG, SHORT, m=m, m_meta=meta)]
    cfg = al.muon_cfg(lr=1.0, parts=1, scale=al.SCALE_NONE)
    al.muon_step(st, cfg, 1, al.workspace(al.muon_workspace_bytes(st, cfg)))
    for p, want in zip(PICKED, _orthogonal(g, PICKED)):
        off = float((-st[0].param[p].double() - want).norm() / want.norm())
        print(f"from {p.start}: off {off:.1e}", flush=True)
        assert off < 0.05
    for at in (0, 1 << 31, 1 << 32, n - 65536):
        new = ((1.0 - cfg.beta) * g.view(-1)[at : at + 65536].double()).float().view(-1, 256)
        top = new.abs().amax(1, keepdim=True)
        assert torch.equal(meta[at // 256 : at // 256 + 256], top[:, 0])
        y = 127.0 * new.double() / top.double()
        assert (m[at : at + 65536].view(torch.int8).view(-1, 256).double() - y).abs().max() <= 0.5


@pytest.mark.parametrize("tokens,vocab", [(3, LONG + 3), (LONG + 5, 70)])
def test_the_head_loss_past_32_bits(tokens, vocab):
    """A table, and hidden states, of more than 2^32 elements, with targets in the last of them; 1% of each result, as above (bf16 gradients leave 3e-3)."""
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import vocab as voc

    h = torch.empty(tokens, SHORT, device="cuda", dtype=torch.bfloat16).normal_()
    w = torch.empty(vocab, SHORT, device="cuda", dtype=torch.bfloat16).normal_(0, 1.0 / 32)
    target = torch.arange(tokens, device="cuda") % vocab
    if tokens < 10:
        target = torch.tensor([vocab - 1, (1 << 31) // SHORT, (1 << 32) // SHORT], device="cuda")
    loss, dh = torch.empty(tokens, device="cuda"), torch.full((tokens, SHORT), float("nan"), device="cuda", dtype=torch.bfloat16)
    dw = torch.full((vocab, SHORT), float("nan"), device="cuda", dtype=torch.bfloat16)
    voc.linear_xent(h, w, target, loss, al.workspace(voc.linear_xent_workspace_bytes(h, w, dh, dw)), dh=dh, dw=dw)

    def near(got, want, what):
        off = float((got.double() - want).norm() / want.norm())
        print(f"{what}: off {off:.1e}", flush=True)
        assert off < 0.01

    if tokens < 10:
        z = torch.cat([h.double() @ w[p].double().t().contiguous() for p in _parts_of(vocab)], 1)
        d = torch.softmax(z, 1)
        d[torch.arange(3), target] -= 1.0
        near(loss, torch.logsumexp(z, 1) - z[torch.arange(3), target], "loss")
        near(dh, sum(d[:, p] @ w[p].double() for p in _parts_of(vocab)), "dh")
        for p in PICKED + [slice(LONG, vocab)]:
            near(dw[p], d[:, p].t().contiguous() @ h.double(), f"dw from {p.start}")
        assert all(bool(dw[p].isfinite().all()) for p in _parts_of(vocab))
        return
    wide = w.double()
    total = torch.zeros_like(wide)
    for p in _parts_of(tokens):
        z = h[p].double() @ wide.t().contiguous()
        d = torch.softmax(z, 1)
        rows = torch.arange(len(z), device="cuda")
        want = torch.logsumexp(z, 1) - z[rows, target[p]]
        d[rows, target[p]] -= 1.0
        assert (loss[p].double() - want).abs().max() < 1e-3
        total += d.t().contiguous() @ h[p].double()
        assert float((dh[p].double() - d @ wide).norm()) < 0.01 * float((d @ wide).norm())
    near(dw, total, "dw")


def test_the_longest_vocabulary_with_the_most_tokens():
    """2^38 logits of 64 features: passes of the statistics whose grid stays below 2^32 threads, every token's statistics written. Losses within 64 products summed in fp32 (at most
    (64 / 32 + 6) 2^-24 of the sum of magnitudes, twice: lse's and the target's) and the sum of 2^24 exponentials (2^-24 for each of 16 in a lane, 8 a thousand groups and 6 at the end)."""
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import vocab as voc

    tokens, vocab = 16384, 1 << 24
    h = torch.empty(tokens, 64, device="cuda", dtype=torch.bfloat16).normal_()
    w = torch.empty(vocab, 64, device="cuda", dtype=torch.bfloat16).normal_(0, 1.0 / 8)
    target = torch.randint(vocab, (tokens,), device="cuda")
    loss = torch.full((tokens,), float("nan"), device="cuda")
    ws = al.workspace(voc.linear_xent_workspace_bytes(h, w))
    ws.fill_(0xff)
    voc.linear_xent(h, w, target, loss, ws)
    assert bool(loss.isfinite().all())
    picked = torch.cat([torch.arange(0, tokens, 700), torch.arange(tokens - 8, tokens), torch.arange(8188, 8196)]).cuda()
    x = h[picked].double()
    top, total, size = torch.full((len(picked),), -1e300, dtype=torch.float64, device="cuda"), 0.0, 0.0
    for p in _parts_of(vocab, 1 << 20):
        z = x @ w[p].double().t().contiguous()
        new = torch.maximum(top, z.amax(1))
        total = total * (top - new).exp() + (z - new[:, None]).exp().sum(1)
        top = new
        size = max(size, float((x.abs() @ w[p].double().abs().t().contiguous()).max()))
    want = top + total.log() - (x * w[target[picked]].double()).sum(1)
    tol = 2.0**-24 * (2 * 8 * size + 2 * 40 + 300) + 4 * 2.0**-24 * want.abs()
    off = (loss[picked].double() - want).abs()
    print(f"off {float(off.max()):.1e} of {float(tol.min()):.1e}", flush=True)
    assert bool((off <= tol).all())
