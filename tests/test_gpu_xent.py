"""Cross entropy of a linear head and its gradients against the 64-bit definition: sizes from one, pitches, ignored and weighted tokens, pieces of the vocabulary, bases, graphs."""
import numpy as np
import pytest
import torch

from tests.act_util import B16, DT, U, f64, gpu, out_like, untouched

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, tokens, hidden, vocab, seed=0, sharp=1.0, ignored=True, weighted=True, wide=True):
        rng = np.random.default_rng(seed + tokens * 31 + hidden * 7 + vocab)
        b = lambda *s: torch.from_numpy(rng.normal(size=s).astype(np.float32)).bfloat16()  # noqa: E731
        self.h, self.w = b(tokens, hidden), (b(vocab, hidden) * (sharp / hidden**0.5)).bfloat16()
        t = rng.integers(0, vocab, tokens)
        if ignored and tokens > 2:
            t[1::4] = -100
            t[2::9] = vocab
        self.target = torch.from_numpy(t.astype(np.int64 if wide else np.int32))
        self.weight = torch.from_numpy(rng.uniform(0.1, 2.0, tokens).astype(np.float32)) if weighted else None
        self.scale = 1.0 / tokens
        self.keep = (t >= 0) & (t < vocab)

    def exact(self):
        """Losses, lse, d and what the products may be off by, in binary64."""
        h, w = f64(self.h), f64(self.w)
        z = h @ w.T
        top = z.max(1, keepdims=True)
        lse = np.log(np.exp(z - top).sum(1, keepdims=True)) + top
        t = np.where(self.keep, self.target.numpy(), 0)
        rows = np.arange(len(t))
        loss = np.where(self.keep, lse[:, 0] - z[rows, t], 0.0)
        coef = np.float64(np.float32(self.scale)) * (1.0 if self.weight is None else self.weight.numpy().astype(np.float64)) * self.keep
        d = np.exp(z - lse)
        d[rows, t] -= 1.0
        # a logit: hidden products summed in fp32 (hidden / 32 matrix instructions one after the other, 5 levels in one), as a share of the sum of magnitudes
        off_z = (h.shape[1] / 32 + 6) * U * (np.abs(h) @ np.abs(w).T).max(1)
        # exp: x log2(e) rounded, times |x| log(2), and the hardware's exp2 to 2 units; lse besides: the sums of sums, log and max of vocab terms
        span = np.abs(z - lse).max(1)
        off_lse = off_z + (np.log2(max(2, w.shape[0])) + 8) * U * (1 + np.abs(lse[:, 0])) + span * 2 * U
        off_p = off_z + off_lse + (span + 4) * 2 * U  # relative, of exp(z - lse)
        return h, w, loss, lse[:, 0], coef, d, off_z + off_lse, off_p


def call(c, dh=None, dw=None, base=None, lse=False, pad=(0, 0), loss=True):
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import vocab as voc

    h, w = gpu(c.h, pad=pad[0], shift=pad[0]), gpu(c.w, pad=pad[1])
    tokens, hidden = c.h.shape
    out = dict(loss=torch.full((tokens,), float("nan"), device="cuda") if loss else None, lse=torch.full((tokens,), float("nan"), device="cuda") if lse else None)
    whole = None
    if dh:
        out["dh"], whole = out_like(tokens, hidden, DT[dh], pad=3, shift=2)
    if dw:
        out["dw"] = torch.full(c.w.shape, float("nan"), dtype=DT[dw], device="cuda")
    ws = al.workspace(voc.linear_xent_workspace_bytes(h, w, out.get("dh"), out.get("dw")))
    ws.fill_(0xff)
    weight = None if c.weight is None else c.weight.cuda()
    voc.linear_xent(h, w, c.target.cuda(), out["loss"], ws, weight=weight, scale=c.scale, lse=out["lse"], dh=out.get("dh"), dw=out.get("dw"), base=base)
    torch.cuda.synchronize()
    if whole is not None:
        assert untouched(out["dh"], whole)
    return out


def check(c, out, dh=None, dw=None, base=None):
    h, w, loss, lse, coef, d, off_loss, off_p = c.exact()
    if out["loss"] is not None:
        assert (np.abs(f64(out["loss"]) - loss) <= off_loss + 2 * U * np.abs(loss)).all()
    if out["lse"] is not None:
        assert (np.abs(f64(out["lse"]) - np.where(c.keep, lse, 0.0)) <= off_loss + 2 * U * np.abs(lse)).all()
    p = np.where(d < 0, d + 1.0, d)  # the target's probability where it was taken off
    e = d * coef[:, None]
    # d: the probability's error, its subtraction and product, and the rounding of the parts
    off_e = (p * off_p[:, None] + 4 * U * np.abs(d)) * np.abs(coef)[:, None]
    for name, kind in (("dh", dh), ("dw", dw)):
        if not kind:
            continue
        part = off_e + np.abs(e) * (B16 if kind == "bf16" else B16**2 + U)
        a, x, k = (part, w, w.shape[0]) if name == "dh" else (part.T, h, h.shape[0])
        m = np.abs(e) if name == "dh" else np.abs(e).T
        want = (e @ w) if name == "dh" else e.T @ h
        tol = a @ np.abs(x) + (k / 32 + 12) * U * (m @ np.abs(x))
        if name == "dw" and base is not None:
            want = want + base
            tol = tol + U * np.abs(base)
        tol = tol + np.abs(want) * (B16 if kind == "bf16" else 2 * U)
        got = f64(out[name])
        assert (np.abs(got - want) <= tol * 1.01 + 1e-30).all(), (name, np.abs(got - want).max(), (np.abs(got - want) / (tol + 1e-30)).max())


SIZES = [(1, 8, 1), (1, 1, 2), (2, 3, 5), (3, 64, 64), (17, 65, 63), (64, 128, 130), (70, 100, 257), (130, 72, 1000), (257, 264, 300), (300, 1001, 777)]


@pytest.mark.parametrize("tokens,hidden,vocab", SIZES)
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_against_the_definition(tokens, hidden, vocab, kind):
    c = Case(tokens, hidden, vocab, wide=kind == "f32")
    check(c, call(c, kind, kind, lse=True), kind, kind)
    check(c, call(c, kind, kind, pad=(5, 8)), kind, kind)
    check(c, call(c, kind, kind, pad=(1, 3)), kind, kind)


@pytest.mark.parametrize("dh,dw", [(None, None), ("bf16", None), (None, "f32"), ("bf16", "f32"), ("f32", "bf16")])
def test_what_is_asked_for(dh, dw):
    c = Case(90, 200, 500)
    out = call(c, dh, dw, loss=dh != "f32")
    check(c, out, dh, dw)


@pytest.mark.parametrize("sharp", [0.0, 8.0, 60.0])
def test_flat_and_sharp_distributions(sharp):
    """All logits equal, and probabilities of one and of nothing."""
    c = Case(65, 96, 700, sharp=sharp)
    check(c, call(c, "f32", "f32"), "f32", "f32")
    check(c, call(c, "bf16", "bf16"), "bf16", "bf16")


def test_large_logits():
    """Logits of thousands: the maximum is taken off first."""
    c = Case(40, 64, 300, sharp=3000.0, ignored=False)
    out = call(c, "f32", "f32")
    assert out["loss"].isfinite().all() and out["dh"].isfinite().all() and out["dw"].isfinite().all()
    check(c, out, "f32", "f32")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_pieces_of_the_vocabulary(kind):
    """Tokens times vocabulary past 2^26: several pieces, dh summed over them, a last piece that is no multiple of a tile."""
    c = Case(2100, 40, 33001, ignored=True)
    check(c, call(c, kind, kind), kind, kind)


def test_a_block_of_statistics_past_its_tokens():
    """More than 16384 tokens: the statistics go in two blocks."""
    c = Case(16500, 16, 90)
    check(c, call(c, "bf16", "f32"), "bf16", "f32")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_base_and_in_place(kind):
    c = Case(100, 130, 310)
    base = torch.randn(310, 130, device="cuda").to(DT[kind])
    out = call(c, None, kind, base=base)
    check(c, out, None, kind, f64(base))
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import vocab as voc

    h, w, dw = c.h.cuda(), c.w.cuda(), base.clone()
    ws = al.workspace(voc.linear_xent_workspace_bytes(h, w, None, dw))
    voc.linear_xent(h, w, c.target.cuda(), None, ws, weight=c.weight.cuda(), scale=c.scale, dw=dw, base=dw)
    assert torch.equal(dw, out["dw"])


def test_rows_without_a_target_are_as_if_they_were_not_there():
    """NaN in the hidden state and the weight of an ignored token reaches neither gradients nor other losses; its own are zero."""
    c = Case(70, 64, 200)
    c.h[~c.keep] = float("nan")
    c.weight[~torch.from_numpy(c.keep)] = float("nan")
    out = call(c, "f32", "f32", lse=True)
    assert out["dw"].isfinite().all()
    for name in ("loss", "lse", "dh"):
        assert out[name].isfinite().all() and not out[name][torch.from_numpy(~c.keep)].any()
    c.h[~c.keep], c.weight[~torch.from_numpy(c.keep)] = 0.0, 0.0
    check(c, out, "f32", "f32")


def test_no_target_at_all_and_no_tokens():
    c = Case(20, 64, 100)
    c.target.fill_(-1)
    out = call(c, "f32", "bf16")
    assert not out["loss"].any() and not out["dh"].any() and not out["dw"].any()
    from paper_2608_22322_amd import vocab as voc

    base, dw = torch.randn(100, 64, device="cuda"), torch.empty(100, 64, device="cuda")
    none = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    voc.linear_xent(none, c.w.cuda(), torch.empty(0, dtype=torch.long, device="cuda"), None, None, dw=dw, base=base)
    assert torch.equal(dw, base)


def test_bad_values_show():
    c = Case(30, 64, 100, ignored=False)
    c.h[3, 5] = float("nan")
    out = call(c, "f32", "f32")
    assert out["loss"][3].isnan() and out["dh"][3].isnan().all() and out["dw"].isnan().any()
    assert out["loss"][torch.arange(30) != 3].isfinite().all()


def test_gradient_against_differences():
    """The loss of the 64-bit definition, moved along a direction: the directional derivative that the kernel's gradients give. The definition's
    curvature is at most |v|^2 sum |coef| max |w|^2, so a step of 1e-5 leaves 1e-10 of that; the gradients' own error is check()'s."""
    c = Case(50, 48, 120)
    out = call(c, "f32", "f32")
    h, w, _, _, coef, _, _, _ = c.exact()
    t = np.where(c.keep, c.target.numpy(), 0)

    def total(h, w):
        z = h @ w.T
        top = z.max(1, keepdims=True)
        return float((coef * (np.log(np.exp(z - top).sum(1)) + top[:, 0] - z[np.arange(len(t)), t])).sum())

    rng = np.random.default_rng(1)
    for name, x in (("dh", h), ("dw", w)):
        v = rng.normal(size=x.shape)
        e = 1e-5
        moved = [(h + s * v, w) if name == "dh" else (h, w + s * v) for s in (e, -e)]
        slope = (total(*moved[0]) - total(*moved[1])) / (2 * e)
        got = float((f64(out[name]) * v).sum())
        # bf16 parts: 2^-16 of each product's magnitude; the differences: 1e-10 times third derivatives of the order of |v|^3 |w|^3 sum coef
        size = np.abs(f64(out[name]) * v).sum()
        assert abs(got - slope) <= size * 2.0**-12 + 1e-7


def test_repeats_bit_for_bit():
    c = Case(200, 128, 900)
    a, b = call(c, "bf16", "f32"), call(c, "bf16", "f32")
    assert all(torch.equal(a[k], b[k]) for k in ("loss", "dh", "dw"))


def test_replayed_graphs_that_share_a_workspace():
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import vocab as voc

    made = []
    for tokens, vocab in ((100, 400), (300, 90)):
        c = Case(tokens, 64, vocab)
        h, w, t = c.h.cuda(), c.w.cuda(), c.target.cuda()
        made.append((h, w, t, torch.empty(tokens, device="cuda"), torch.empty(tokens, 64, device="cuda"), torch.empty(vocab, 64, device="cuda")))
    ws = al.workspace(max(voc.linear_xent_workspace_bytes(m[0], m[1], m[4], m[5]) for m in made))
    for h, w, t, loss, dh, dw in made:
        voc.linear_xent(h, w, t, loss, ws, dh=dh, dw=dw)
    torch.cuda.synchronize()
    graphs = []
    for h, w, t, loss, dh, dw in made:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            voc.linear_xent(h, w, t, loss, ws, dh=dh, dw=dw)
        graphs.append(g)
    for seed in range(3):
        torch.manual_seed(seed)
        for m in made:
            m[0].copy_(torch.randn_like(m[0]))
            m[2].random_(-1, m[1].shape[0])
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for h, w, t, loss, dh, dw in made:
            got = loss.clone(), dh.clone(), dw.clone()
            voc.linear_xent(h, w, t, loss, ws, dh=dh, dw=dw)
            assert all(torch.equal(x, y) for x, y in zip(got, (loss, dh, dw)))


@pytest.mark.parametrize("pad,tokens", [(0, 1), (0, 70), (8, 130), (4, 65), (0, 16450)])
def test_hidden_states_read_where_they_are(pad, tokens):
    """Without dw and with whole, aligned rows h is not copied: what an ignored token holds still reaches nothing, and other pitches give the same."""
    c = Case(tokens, 128, 90 if tokens > 1000 else 300)
    c.h[~c.keep] = float("nan")
    out = call(c, "f32", None, lse=True, pad=(pad, 0))
    only = call(c, None, None, pad=(pad, 0))
    assert torch.equal(only["loss"], out["loss"])
    packed = call(c, "f32", "f32", lse=True, pad=(pad, 0))  # dw: h is copied
    for name in ("loss", "lse", "dh"):
        assert out[name].isfinite().all() and not out[name][torch.from_numpy(~c.keep)].any()
        assert torch.equal(out[name], packed[name])
    c.h[~c.keep] = 0.0
    check(c, out, "f32")


def test_streams_and_two_calls_at_once():
    """Two calls on streams of their own with workspaces of their own, at the same time."""
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import vocab as voc

    cases = [Case(300, 128, 2000), Case(500, 200, 1500)]
    want = [call(c, "f32", "f32") for c in cases]
    made = []
    for c in cases:
        h, w, t = c.h.cuda(), c.w.cuda(), c.target.cuda()
        dh, dw = torch.empty(c.h.shape, device="cuda"), torch.empty(c.w.shape, device="cuda")
        made.append((h, w, t, c.weight.cuda(), torch.empty(len(t), device="cuda"), dh, dw, al.workspace(voc.linear_xent_workspace_bytes(h, w, dh, dw)), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(3):
        for c, (h, w, t, weight, loss, dh, dw, ws, st) in zip(cases, made):
            voc.linear_xent(h, w, t, loss, ws, weight=weight, scale=c.scale, dh=dh, dw=dw, stream=st)
    torch.cuda.synchronize()
    for (_, _, _, _, loss, dh, dw, _, _), x in zip(made, want):
        assert torch.equal(loss, x["loss"]) and torch.equal(dh, x["dh"]) and torch.equal(dw, x["dw"])


@pytest.mark.parametrize("tokens,hidden,vocab", [(3, 1 << 18, 5), (2, 100001, 70), (70, 8, 1 << 20), (1, 3, 300007), (5, 16, (1 << 21) + 3)])
def test_long_sides(tokens, hidden, vocab):
    """Features or a vocabulary far longer than the other sides."""
    c = Case(tokens, hidden, vocab, ignored=False)
    check(c, call(c, "f32", "bf16", lse=True), "f32", "bf16")
    check(c, call(c), None, None)
