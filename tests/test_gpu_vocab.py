"""Embeddings and their gradient against exact sums: types, ids, repeated and frequent ones, pitches, bases, offsets past 32 bits, graphs."""
import numpy as np
import pytest
import torch

from tests.act_util import B16, DT, U, f64, gpu, out_like, untouched

pytestmark = pytest.mark.gpu

UNIT = {"f32": U, "bf16": B16}


def ids_of(kind, tokens, vocab, seed, wide=True):
    rng = np.random.default_rng(seed)
    if kind == "random":
        x = rng.integers(0, vocab, tokens)
    elif kind == "few":
        x = rng.integers(0, min(vocab, 3), tokens)
    elif kind == "one":
        x = np.full(tokens, vocab - 1)
    elif kind == "descending":
        x = (tokens - 1 - np.arange(tokens)) % vocab
    else:  # "ignored": ids below 0 and from vocab on among the others
        x = rng.integers(-2, vocab + 2, tokens)
        x[::7] = -100
    return torch.from_numpy(x.astype(np.int64 if wide else np.int32))


@pytest.mark.parametrize("tokens,vocab,cols", [(1, 1, 1), (1, 5, 4096), (7, 3, 5), (300, 50, 1001), (65, 10, 512), (513, 4, 520), (10, 10, 3)])
@pytest.mark.parametrize("table,out", [("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_lookup(tokens, vocab, cols, table, out):
    from paper_2608_22322_amd import vocab as voc

    w = torch.from_numpy(np.random.default_rng(cols).normal(size=(vocab, cols)).astype(np.float32)).to(DT[table])
    for wide in (True, False):
        ids = ids_of("ignored", tokens, vocab, tokens, wide)
        view, buf = out_like(tokens, cols, DT[out], pad=5, shift=3)
        voc.embed_forward(gpu(w, pad=3, shift=1), ids.cuda(), view, scale=1.7)
        s = np.float32(1.7)
        rows = f64(w) * np.float64(s)
        ok = (ids >= 0) & (ids < vocab)
        want = np.where(ok.numpy()[:, None], rows[ids.clamp(0, vocab - 1).numpy()], 0.0)
        # the product in fp32, then the rounding to the output's type
        assert (np.abs(f64(view) - want) <= np.abs(want) * (U + (B16 if out == "bf16" else 0)) * 1.01).all()
        assert not f64(view)[~ok.numpy()].any()
        assert untouched(view, buf)


def backward(dy, ids, vocab, grad, scale=1.0, base=None, dw=None):
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import vocab as voc

    dw = torch.full((vocab, dy.shape[1]), float("nan"), dtype=grad, device="cuda") if dw is None else dw
    ws = al.workspace(voc.embed_backward_workspace_bytes(dy, dw))
    ws.fill_(0xff)
    voc.embed_backward(dy, ids, dw, ws, scale=scale, base=base)
    return dw


def check_sums(got, dy, ids, vocab, unit, scale, base):
    """Sums of n numbers in fp32, pieces first: at most n + 2 roundings of the sum of magnitudes, one each for scale and base, one to the output's type."""
    x, t = f64(dy), ids.cpu().numpy().astype(np.int64)
    ok = (t >= 0) & (t < vocab)
    want, mag, n = np.zeros((vocab, x.shape[1])), np.zeros((vocab, x.shape[1])), np.bincount(t[ok], minlength=vocab)
    np.add.at(want, t[ok], x[ok])
    np.add.at(mag, t[ok], np.abs(x[ok]))
    s = np.float64(np.float32(scale))
    b = 0.0 if base is None else base
    want, mag = want * s + b, mag * abs(s) + np.abs(b)
    tol = mag * (n[:, None] + 4) * U + np.abs(want) * unit
    assert (np.abs(got - want) <= tol).all(), np.abs(got - want).max()


@pytest.mark.parametrize("kind", ["random", "few", "one", "descending", "ignored"])
@pytest.mark.parametrize("tokens,vocab,cols", [(1, 1, 1), (2, 9, 3), (31, 7, 64), (33, 5, 100), (300, 500, 1001), (1024, 40, 36), (1025, 40, 1028), (3000, 2100, 50),
                                               (4097, 11, 130)])
def test_gradient(kind, tokens, vocab, cols):
    rng = np.random.default_rng(tokens)
    for dtype, grad, wide, with_base in (("f32", "f32", True, False), ("bf16", "bf16", False, True), ("bf16", "f32", True, True), ("f32", "bf16", False, False)):
        dy = torch.from_numpy(rng.normal(size=(tokens, cols)).astype(np.float32)).to(DT[dtype])
        ids = ids_of(kind, tokens, vocab, cols, wide).cuda()
        base = torch.from_numpy(rng.normal(size=(vocab, cols)).astype(np.float32)).to(DT[grad]).cuda() if with_base else None
        held = gpu(dy, pad=3, shift=1)
        got = backward(held, ids, vocab, DT[grad], 0.3, base)
        check_sums(f64(got), dy, ids, vocab, UNIT[grad], 0.3, None if base is None else f64(base))
        if with_base:  # in place: the same values
            assert torch.equal(backward(held, ids, vocab, DT[grad], 0.3, base=base, dw=base), got)


def test_rows_without_a_token_are_left_alone_in_place():
    dw = torch.full((50, 70), float("nan"), device="cuda")
    dw[7] = 1.0
    got = backward(torch.ones(3, 70, device="cuda"), torch.tensor([7, -1, 7], device="cuda"), 50, torch.float32, base=dw, dw=dw)
    assert (got[7] == 3.0).all() and got[:7].isnan().all() and got[8:].isnan().all()


def test_what_a_token_without_an_id_holds_is_not_read_into_sums():
    dy = torch.ones(200, 40, device="cuda")
    ids = torch.arange(200, device="cuda") % 9
    ids[::3], dy[::3] = -100, float("nan")
    assert backward(dy, ids, 9, torch.float32).isfinite().all()


def test_many_tokens_merge_twice():
    """More than 64 runs of 1024: a second merge; order kept within an id, so the result repeats bit for bit."""
    tokens, vocab = 150001, 977
    g = torch.Generator(device="cuda").manual_seed(3)
    dy = torch.empty(tokens, 12, device="cuda").normal_(generator=g)
    ids = torch.randint(-1, vocab, (tokens,), device="cuda", generator=g)
    a = backward(dy, ids, vocab, torch.float32)
    check_sums(f64(a), dy, ids, vocab, U, 1.0, None)
    assert torch.equal(a, backward(dy, ids.int(), vocab, torch.float32))


def test_exact_integers_whatever_the_order():
    """Small whole numbers: every sum is exact, so it has to be equal."""
    tokens, vocab, cols = 20000, 300, 24
    g = torch.Generator(device="cuda").manual_seed(4)
    dy = torch.randint(-8, 9, (tokens, cols), device="cuda", generator=g).float()
    ids = (torch.randint(0, vocab, (tokens,), device="cuda", generator=g).float() ** 2 / vocab).long()
    want = torch.zeros(vocab, cols, dtype=torch.float64, device="cuda").index_add_(0, ids, dy.double())
    assert torch.equal(backward(dy.bfloat16(), ids, vocab, torch.float32).double(), want)


def test_a_vocabulary_past_the_narrow_keys():
    """From 2^22 ids on the sort's keys are 64 bits."""
    vocab, tokens = (1 << 22) + 5, 3000
    g = torch.Generator(device="cuda").manual_seed(5)
    ids = torch.randint(0, vocab, (tokens,), device="cuda", generator=g)
    ids[:50], ids[50:60] = vocab - 1, 0
    dy = torch.randint(-8, 9, (tokens, 4), device="cuda", generator=g).float()
    got = backward(dy, ids, vocab, torch.float32)
    assert torch.equal(got.double(), torch.zeros(vocab, 4, dtype=torch.float64, device="cuda").index_add_(0, ids, dy.double()))


def test_offsets_past_32_bits():
    """Rows at the end of a table of more than 2^32 bytes, looked up and summed."""
    from paper_2608_22322_amd import vocab as voc

    vocab, cols = 600000, 4096
    table = torch.zeros(vocab, cols, dtype=torch.bfloat16, device="cuda")
    table[-1], table[-2] = 3.0, 5.0
    ids = torch.tensor([vocab - 1, vocab - 2, 0], device="cuda")
    out = torch.empty(3, cols, dtype=torch.bfloat16, device="cuda")
    voc.embed_forward(table, ids, out)
    assert (out[0] == 3).all() and (out[1] == 5).all() and not out[2].any()
    backward(out, ids, vocab, torch.bfloat16, base=table, dw=table)
    assert (table[-1] == 6).all() and (table[-2] == 10).all() and not table[: vocab - 2].any()


def test_no_tokens():
    base = torch.randn(5, 7, device="cuda")
    none = torch.empty(0, dtype=torch.long, device="cuda")
    assert torch.equal(backward(torch.empty(0, 7, device="cuda"), none, 5, torch.float32, base=base), base)
    assert not backward(torch.empty(0, 7, device="cuda"), none, 5, torch.float32).any()


def test_replayed_graphs_that_share_a_workspace():
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import vocab as voc

    g = torch.Generator(device="cuda").manual_seed(6)
    dy = [torch.empty(n, 40, device="cuda") for n in (3000, 500)]
    ids = [torch.empty(n, dtype=torch.long, device="cuda") for n in (3000, 500)]
    dw = [torch.empty(60, 40, device="cuda") for _ in dy]
    ws = al.workspace(max(voc.embed_backward_workspace_bytes(d, w) for d, w in zip(dy, dw)))

    def fill():
        for d, i in zip(dy, ids):
            d.normal_(generator=g)
            i.random_(-1, 60, generator=g)

    fill()
    for d, i, w in zip(dy, ids, dw):
        voc.embed_backward(d, i, w, ws)
    torch.cuda.synchronize()
    graphs = []
    for d, i, w in zip(dy, ids, dw):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            voc.embed_backward(d, i, w, ws)
        graphs.append(graph)
    for _ in range(3):
        fill()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for d, i, w in zip(dy, ids, dw):
            assert torch.equal(w, backward(d, i, 60, torch.float32))


def test_streams():
    """On a side stream, given or current, as on the default one."""
    from paper_2608_22322_amd import vocab as voc

    ids = ids_of("ignored", 700, 90, 8).cuda()
    table, dy = torch.randn(90, 100, device="cuda"), torch.randn(700, 100, device="cuda")
    out = [torch.empty(700, 100, device="cuda") for _ in range(3)]
    want = backward(dy, ids, 90, torch.float32)
    voc.embed_forward(table, ids, out[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    voc.embed_forward(table, ids, out[1], stream=side)
    with torch.cuda.stream(side):
        voc.embed_forward(table, ids, out[2])
        got = backward(dy, ids, 90, torch.float32)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2]) and torch.equal(got, want)


@pytest.mark.parametrize("vocab", [(1 << 22) - 1, 1 << 22])
def test_both_sides_of_the_narrow_keys(vocab):
    """The last id and one past it, at the largest vocabulary whose keys are 32 bits and the next."""
    ids = torch.tensor([vocab - 1, vocab, 0, vocab - 1, -1, vocab - 2] * 200, device="cuda")
    got = backward(torch.ones(1200, 2, device="cuda"), ids, vocab, torch.float32)
    assert (got[-1] == 400).all() and (got[0] == 200).all() and (got[-2] == 200).all() and float(got.sum()) == 1600


@pytest.mark.parametrize("tokens,vocab,cols", [(3, 4, (1 << 20) + 3), (70, 1, 100001), (40, 1 << 20, 1)])
def test_long_sides(tokens, vocab, cols):
    from paper_2608_22322_amd import vocab as voc

    ids = ids_of("random", tokens, vocab, 3).cuda()
    dy = torch.randint(-8, 9, (tokens, cols), device="cuda").float()
    got = backward(dy.bfloat16(), ids, vocab, torch.float32)
    assert torch.equal(got.double(), torch.zeros(vocab, cols, dtype=torch.float64, device="cuda").index_add_(0, ids, dy.double()))
    out = torch.empty(tokens, cols, device="cuda")
    voc.embed_forward(got, ids, out)
    assert torch.equal(out, got[ids])
