"""The orthogonalised momentum step: codes and metadata against the code's definition, parameters against the 64-bit step, lists of many shapes."""
import numpy as np
import pytest
import torch

import oracle
from tests.act_util import f64
from tests.gpu_util import compare_bits, compare_codes, to_np
from tests.ortho_util import newton_schulz, tolerance

pytestmark = pytest.mark.gpu


def states(shapes, uf8, grad_bf16, seed, momentum=True):
    import paper_2608_22322_amd as al

    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for r, c in shapes:
        p = torch.empty(r, c, device="cuda").normal_(0, 0.02, generator=g)
        grad = torch.empty(r, c, device="cuda").normal_(0, 1e-3, generator=g)
        grad = grad.bfloat16() if grad_bf16 else grad
        m, meta = al.alloc_state(r * c, al.Spec(al.UF8 if uf8 else al.FP32, 256))
        if momentum and r * c:
            start = torch.empty(r * c, device="cuda").normal_(0, 5e-4, generator=g)
            if uf8:
                al.quantize(al.UF8, start, 256, 0.0, m, meta)
            else:
                m.copy_(start)
        out.append(al.ParamState(p, grad, r, c, m=m, m_meta=meta))
    return out


def expected(st, cfg, uf8):
    """(m, u, parameters, allowed error of the parameters) of a step in binary64 from the state's buffers; codes are made by the caller."""
    n = st.rows * st.cols
    if uf8:
        m = oracle.State(oracle.UF8, n, 256)
        m.codes[:] = to_np(st.m)[: m.codes.size]
        m.meta[:] = to_np(st.m_meta)[: m.meta.size]
        old = m.decode().astype(np.float64)
    else:
        old = to_np(st.m)[:n].astype(np.float64)
    g = f64(st.grad).reshape(-1)
    beta = cfg.beta
    m = (beta * old + (1.0 - beta) * g).astype(np.float32)
    u = (beta * m.astype(np.float64) + (1.0 - beta) * g).astype(np.float32) if cfg.nesterov else m
    k = cfg.ortho
    want, seen = newton_schulz(u.reshape(st.rows, st.cols), k.steps, (k.a, k.b, k.c), k.eps)
    scale = {0: 1.0, 1: max(1.0, st.rows / st.cols) ** 0.5, 2: 0.2 * max(st.rows, st.cols) ** 0.5}[cfg.scale]
    p = f64(st.param) * (1.0 - cfg.lr * cfg.weight_decay) - cfg.lr * scale * want
    allowed = cfg.lr * scale * tolerance(seen, k.parts, 2.0**-24, False) + 2.0**-24 * np.sqrt((p * p).sum())
    return m, p, allowed


def check(sts, cfg, uf8):
    import paper_2608_22322_amd as al

    want = [expected(s, cfg, uf8) if s.rows * s.cols else None for s in sts]
    ws = al.workspace(al.muon_workspace_bytes(sts, cfg))
    ws.fill_(0xff)
    al.muon_step(sts, cfg, 1, ws)
    torch.cuda.synchronize()
    for i, (s, w) in enumerate(zip(sts, want)):
        if w is None:
            continue
        m, p, allowed = w
        n = s.rows * s.cols
        off = np.sqrt(((f64(s.param) - p) ** 2).sum())
        assert off <= allowed, (i, s.rows, s.cols, off, allowed)
        if uf8:
            ref = oracle.State(oracle.UF8, n, 256)
            ref.encode(m)
            compare_codes(to_np(s.m)[: ref.codes.size], ref.codes, ref.y, f"tensor {i} m")
            compare_bits(to_np(s.m_meta)[: ref.meta.size], ref.meta, f"tensor {i} meta")
        else:
            compare_bits(to_np(s.m)[:n], m, f"tensor {i} m")


MIXED = [(64, 64), (1, 300), (300, 1), (63, 65), (130, 50), (0, 7), (257, 300), (64, 64), (1, 1), (500, 100)]


@pytest.mark.parametrize("uf8", [True, False])
@pytest.mark.parametrize("grad_bf16", [True, False])
@pytest.mark.parametrize("parts", [1, 2])
def test_a_list_of_shapes(uf8, grad_bf16, parts):
    import paper_2608_22322_amd as al

    cfg = al.muon_cfg(lr=2e-2, weight_decay=0.1, parts=parts, grad_bf16=grad_bf16, m=al.Spec(al.UF8 if uf8 else al.FP32, 256))
    check(states(MIXED, uf8, grad_bf16, 3), cfg, uf8)


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("scale", [0, 1, 2])
def test_scales_and_momentum(nesterov, scale):
    import paper_2608_22322_amd as al

    cfg = al.muon_cfg(lr=1e-2, beta=0.8, nesterov=nesterov, scale=scale, steps=3, grad_bf16=False)
    check(states([(200, 50), (50, 200), (70, 70)], True, False, 5), cfg, True)


def test_more_matrices_than_share_launches():
    import paper_2608_22322_amd as al

    shapes = [(40 + i % 5, 30 + i % 7) for i in range(70)]
    check(states(shapes, True, True, 9), al.muon_cfg(lr=1e-2), True)


def test_steps_one_after_another_and_parts_of_the_list():
    """Three steps from a fresh state; a part of the list fits the list's workspace, and steps as it does in the list."""
    import paper_2608_22322_amd as al

    shapes = [(120, 300), (300, 120), (64, 1000), (200, 200)]
    a, b = states(shapes, True, True, 11, momentum=False), states(shapes, True, True, 11, momentum=False)
    cfg = al.muon_cfg(lr=1e-2)
    need = al.muon_workspace_bytes(a, cfg)
    ws = al.workspace(need)
    for t in range(1, 4):
        al.muon_step(a, cfg, t, ws)
        for part in (b[:1], b[1:]):
            assert al.muon_workspace_bytes(part, cfg) <= need
            al.muon_step(part, cfg, t, ws)
    for x, y in zip(a, b):  # (parameters: the cut of the products goes by the group, sums in another order)
        assert torch.equal(x.m, y.m) and torch.equal(x.m_meta, y.m_meta)


def test_replayed_in_a_graph():
    import paper_2608_22322_amd as al

    shapes = [(120, 300), (300, 120), (64, 1000)]
    a, b = states(shapes, True, True, 13), states(shapes, True, True, 13)
    cfg = al.muon_cfg(lr=1e-2)
    ws = al.workspace(al.muon_workspace_bytes(a, cfg))
    arr = al.tensor_array(a)
    al.muon_step(a, cfg, 1, ws, arr=arr)
    al.muon_step(b, cfg, 1, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        al.muon_step(a, cfg, 2, ws, arr=arr)
    for t in range(2, 5):
        g.replay()
        torch.cuda.synchronize()
        al.muon_step(b, cfg, t, ws)
        torch.cuda.synchronize()
        for x, y in zip(a, b):
            assert torch.equal(x.param, y.param) and torch.equal(x.m, y.m) and torch.equal(x.m_meta, y.m_meta)


def test_a_zero_gradient_leaves_the_parameters():
    import paper_2608_22322_amd as al

    sts = states([(100, 60)], True, True, 15, momentum=False)
    sts[0].grad.zero_()
    before = sts[0].param.clone()
    cfg = al.muon_cfg(lr=1e-2, eps=0.0)
    al.muon_step(sts, cfg, 1, al.workspace(al.muon_workspace_bytes(sts, cfg)))
    assert torch.equal(sts[0].param, before) and not sts[0].m.any()


def test_step_of_a_named_list():
    """MuonStep: block matrices by their orthogonalised momentum, the rest by AdamW."""
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd.muon import MuonStep

    def make():
        g = torch.Generator(device="cuda").manual_seed(1)
        out = []
        for r, c in ((300, 64), (64, 64), (1, 64), (100, 64)):
            out.append(al.ParamState(torch.empty(r, c, device="cuda").normal_(generator=g), torch.empty(r, c, device="cuda").normal_(generator=g).bfloat16(), r, c))
        return out

    names = ["embed", "layer0.q", "layer0.attn_norm", "layer0.gate"]
    a, b = make(), make()
    opt = MuonStep(a, names)
    for t in (1, 2):
        opt.step(t)
    m = al.Spec(al.UF8, 256)
    for i in (1, 3):
        b[i].m, b[i].m_meta = al.alloc_state(b[i].rows * 64, m)
    v = al.Spec(al.AL8, 256, al.log2_floor_of(1e-16))
    for i in (0, 2):
        b[i].m, b[i].m_meta = al.alloc_state(b[i].rows * 64, m)
        b[i].v, b[i].v_meta = al.alloc_state(b[i].rows * 64, v)
    mats, rest = [b[1], b[3]], [b[0], b[2]]
    mc, ac = al.muon_cfg(), al.adamw_cfg(lr=1e-3, weight_decay=0.0)
    for t in (1, 2):
        al.muon_step(mats, mc, t, al.workspace(al.muon_workspace_bytes(mats, mc)))
        al.adamw_step(rest, ac, t, al.workspace(al.adamw_workspace_bytes(rest, ac)))
    for x, y in zip(a, b):
        assert torch.equal(x.param, y.param)


def test_lists_of_one_kind():
    """MuonStep over matrices alone and over nothing for it to orthogonalise."""
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd.muon import MuonStep

    for names, shapes in ((["layer0.q", "layer1.q"], [(70, 64), (64, 130)]), (["embed", "norm"], [(30, 64), (1, 64)])):
        sts = [al.ParamState(torch.ones(r, c, device="cuda"), torch.randn(r, c, device="cuda").bfloat16(), r, c) for r, c in shapes]
        MuonStep(sts, names).step(1)
        assert all(s.param.isfinite().all() and not (s.param == 1).all() for s in sts)


def test_a_bad_gradient_stays_with_its_matrix():
    import paper_2608_22322_amd as al

    for bad in (float("nan"), float("inf")):
        a, b = (states([(100, 60), (64, 300), (300, 64)], True, False, 17) for _ in range(2))
        a[1].grad[3, 7] = bad
        cfg = al.muon_cfg(lr=1e-2, grad_bf16=False)
        for s in (a, b):
            al.muon_step(s, cfg, 1, al.workspace(al.muon_workspace_bytes(s, cfg)))
        assert a[1].param.isnan().all()
        for i in (0, 2):
            assert torch.equal(a[i].param, b[i].param) and torch.equal(a[i].m, b[i].m)


def test_resumed_from_a_checkpoint(tmp_path):
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import checkpoint

    shapes = [(120, 300), (64, 70)]
    a, b = states(shapes, True, True, 19), states(shapes, True, True, 23)
    cfg = al.muon_cfg(lr=1e-2)
    ws = al.workspace(al.muon_workspace_bytes(a, cfg))
    specs = [{"m": al.Spec(al.UF8, 256)}] * 2
    al.muon_step(a, cfg, 1, ws)
    path = str(tmp_path / "muon.safetensors")
    checkpoint.save(path, a, specs, ["layer0.q", "layer0.k"], "muon", 1)
    for x, y in zip(a, b):
        y.param.copy_(x.param)
        y.grad.copy_(x.grad)
    assert checkpoint.load(path, b, specs, "muon") == ("muon", 1)
    for s in (a, b):
        al.muon_step(s, cfg, 2, ws)
    for x, y in zip(a, b):
        assert torch.equal(x.param, y.param) and torch.equal(x.m, y.m) and torch.equal(x.m_meta, y.m_meta)


@pytest.mark.parametrize("parts", [1, 2])
def test_a_layer(parts):
    """Matrices at whose sizes the wide tiles are taken and steps go two at a time, among small ones: parameters from zero, against the 64-bit form and the same
    roundings in another order (as for the products alone)."""
    import paper_2608_22322_amd as al
    from tests.ortho_util import rounded

    shapes = [(2048, 2048), (256, 2048), (5632, 2048), (2048, 5632), (64, 64), (4224, 4200)]
    sts = states(shapes, False, False, 29, momentum=False)
    for s in sts:
        s.param.zero_()
    cfg = al.muon_cfg(lr=1.0, beta=0.0, nesterov=False, scale=al.SCALE_NONE, parts=parts, grad_bf16=False, m=al.Spec(al.FP32, 256))
    al.muon_step(sts, cfg, 1, al.workspace(al.muon_workspace_bytes(sts, cfg)))
    a, b, c = al.ORTHO_COEFS
    for s in sts:
        wide = s.grad if s.rows <= s.cols else s.grad.t().contiguous()
        got = -(s.param if s.rows <= s.cols else s.param.t()).double()
        y = wide.double() / (wide.double().norm() + 1e-7)
        for _ in range(5):
            q = y @ y.t().contiguous()
            y = a * y + (b * q + c * (q @ q)) @ y
        off = float((got - y).norm() / y.norm())
        like = max(float((rounded(wide, parts, pairs).double() - y).norm() / y.norm()) for pairs in (False, True))
        print(f"{s.rows} x {s.cols}, {parts} parts: off {off:.2e}, its roundings {like:.2e}", flush=True)
        assert off <= like * (1.5 if parts == 1 else 3.0)
