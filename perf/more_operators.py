"""The two ends of a token model and the step of the matrices between them, as cases that can be timed and compared.

The operators: orthogonalising a matrix by Newton-Schulz products, the momentum step that orthogonalises its update (8-bit or
fp32 momentum), the lookup of token embeddings and its gradient, and softmax cross entropy of a linear head with its
gradients. Widths are those of the repository's 1.1B and 7B lists (2048 / 5632 / 256 and 4096 / 11008, 32000 tokens) and its odd
test widths (500, 700, 1001, 1750); token counts run from one token to a batch of four sequences of 2048.

Orthogonalising: X = G / (|G| + eps) with the Frobenius norm, then `steps` times X <- a X + (b A + c A A) X with A = X X^T (or,
for more rows than columns, X <- a X + X (b A + c A A) with A = X^T X).

The momentum step: m <- beta m + (1 - beta) g, u = beta m + (1 - beta) g, p <- p (1 - lr wd) - lr s O(u), O the
orthogonalised u and s = 0.2 sqrt(max(rows, cols)). An 8-bit momentum is, per block of 256 elements, the largest magnitude and
for each element the nearest multiple of a 127th of it; the step computes with m before it is coded.

A token id or a target outside the vocabulary stands for no token: its embedding is zero and it takes part in no gradient or loss.
"""
from __future__ import annotations

import math

import torch

own = False

F32, F64, BF16 = torch.float32, torch.float64, torch.bfloat16
DT = {"fp32": F32, "bf16": BF16}
COEFS = (3.4445, -4.7750, 2.0315)
STEPS, EPS, BETA, BLOCK = 5, 1e-7, 0.95, 256


# ------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a small matrix of a test model: latency is all there is
        dict(name="ortho-500x64", op="ortho", rows=500, cols=64, pad=0, dtype="bf16", out="bf16"),
        # odd sides, fp32 in and out, rows of a wider buffer
        dict(name="ortho-1001x1750", op="ortho", rows=1001, cols=1750, pad=6, dtype="fp32", out="fp32"),
        # the largest matrix of the 7B-wide layer
        dict(name="ortho-4096x11008", op="ortho", rows=4096, cols=11008, pad=0, dtype="bf16", out="bf16"),
        # the step of one layer of the 1.1B model: attention and MLP matrices, 8-bit momentum
        dict(name="muon-layer-2048", op="muon", grad="bf16", momentum="uf8", lr=1e-3, wd=0.1,
             shapes="2048x2048,256x2048,256x2048,2048x2048,5632x2048,5632x2048,2048x5632"),
        # a small model's odd matrices with fp32 gradients and momentum
        dict(name="muon-odd", op="muon", grad="fp32", momentum="fp32", lr=2e-3, wd=0.0, shapes="700x1001,1001x500,500x500,64x1750"),
        # the loss of one token, no gradients: the whole head is read for it
        dict(name="xent-1x4096", op="xent", tokens=1, hidden=4096, vocab=32000, dh="none", dw="none", weight=False, base=False),
        # the head of the 1.1B model over a batch of four sequences, gradients in bf16
        dict(name="xent-8192x2048", op="xent", tokens=8192, hidden=2048, vocab=32000, dh="bf16", dw="bf16", weight=False, base=False),
        # a ragged batch at an odd width and vocabulary, weighted tokens, fp32 gradients added to what earlier microbatches left
        dict(name="xent-1501x1750", op="xent", tokens=1501, hidden=1750, vocab=32003, dh="fp32", dw="fp32", weight=True, base=True),
        # the lookup of one token when a model answers
        dict(name="embed-1x4096", op="embed", tokens=1, hidden=4096, vocab=32000, dtype="fp32", out="bf16", ids="int64"),
        # the lookup of a batch of four sequences
        dict(name="embed-8192x2048", op="embed", tokens=8192, hidden=2048, vocab=32000, dtype="bf16", out="bf16", ids="int64"),
        # its gradient at the 7B width, fp32
        dict(name="dembed-8192x4096", op="dembed", tokens=8192, hidden=4096, vocab=32000, dtype="bf16", grad="fp32", pad=0, ids="int64", base=False),
        # a short ragged batch of an odd-width model, added to the head's gradient of a tied table
        dict(name="dembed-300x1001", op="dembed", tokens=300, hidden=1001, vocab=5003, dtype="fp32", grad="bf16", pad=5, ids="int32", base=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    n = _log_uniform(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.6 else n  # most models round their widths


MOST = 3.1e12  # operations of the largest listed case


def _ns_flops(rows, cols):
    m, n = sorted((rows, cols))
    return STEPS * m * m * (3 * n + m)  # two of the three products are symmetric matrices


def draw(rng):
    op = rng.choice(["ortho", "muon", "xent", "xent", "embed", "dembed"])
    if op == "ortho":
        c = dict(op=op, rows=_width(rng, 16, 8192), cols=_width(rng, 16, 8192), pad=rng.choice([0, 0, 8, 5]),
                 dtype=rng.choice(["bf16", "fp32"]), out=rng.choice(["bf16", "fp32"]))
        while _ns_flops(c["rows"], c["cols"]) * (3 if c["out"] == "fp32" else 1) > MOST:
            c["rows"] = c["rows"] // 2 + 1
        return c
    if op == "muon":
        shapes, left = [], MOST / 3
        for _ in range(rng.randint(1, 5)):
            r, k = _width(rng, 16, 4096), _width(rng, 16, 4096)
            while _ns_flops(r, k) > left:
                r = r // 2 + 1
            left -= _ns_flops(r, k)
            shapes += ["%dx%d" % (r, k)] * rng.choice([1, 1, 2])
            left -= _ns_flops(r, k)
            if left < MOST / 30:
                break
        return dict(op=op, grad=rng.choice(["bf16", "fp32"]), momentum=rng.choice(["uf8", "uf8", "fp32"]),
                    lr=math.exp(rng.uniform(math.log(2e-4), math.log(4e-3))), wd=rng.choice([0.0, 0.1]), shapes=",".join(shapes))
    c = dict(op=op, tokens=_log_uniform(rng, 1, 16384), hidden=_width(rng, 40, 4096), vocab=_width(rng, 300, 50000))
    if op == "xent":
        kind = rng.choice(["none", "bf16", "bf16", "fp32"])
        c.update(dh=kind, dw=kind, weight=rng.random() < 0.5, base=kind != "none" and rng.random() < 0.4)
        while c["tokens"] * c["hidden"] * c["vocab"] * (2 if kind == "none" else 10 if kind == "fp32" else 6) > MOST:
            c["tokens"] = c["tokens"] // 2 + 1
        return c
    c["ids"] = rng.choice(["int64", "int32"])
    if op == "embed":
        c.update(dtype=rng.choice(["fp32", "bf16"]), out=rng.choice(["bf16", "bf16", "fp32"]))
    else:
        c.update(dtype=rng.choice(["fp32", "bf16"]), grad=rng.choice(["fp32", "bf16"]), pad=rng.choice([0, 0, 8, 5]), base=rng.random() < 0.4)
    return c


# ----------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, sigma=1.0):
    return torch.empty(*shape, dtype=F32, device="cuda").normal_(0.0, sigma, generator=g)


def _matrix(g, rows, cols, pad, dtype, sigma=1.0):
    """rows x cols of a buffer of cols + pad columns: normal values, channels whose sizes spread (some run hotter than the rest)."""
    x = _normal(g, rows, cols + pad, sigma=sigma)
    x *= _normal(g, cols + pad, sigma=0.4).exp_()
    return x.to(dtype)[:, :cols]


def _gradient(g, rows, cols, dtype, sigma=1e-3, pad=0):
    """A weight gradient: the product of a few dozen directions that a batch shares, and what its tokens add to them."""
    k = min(rows, cols, 32)
    x = _normal(g, rows, k) @ (_normal(g, k, cols + pad) * (2.0 / math.sqrt(k)))
    x += _normal(g, rows, cols + pad)
    x *= _normal(g, cols + pad, sigma=0.3).exp_() * sigma
    return x.to(dtype)[:, :cols]


def _tokens(g, n, vocab, ignored=0.02):
    """Ids as text has them: the k-th most frequent about as often as 1 / k; a few stand for no token."""
    u = torch.rand(n, device="cuda", dtype=F64, generator=g)
    ids = (torch.exp(u * math.log(vocab + 1)) - 1).long().clamp_(0, vocab - 1)
    spread = ids * 7919 % vocab if vocab % 7919 else ids
    return torch.where(torch.rand(n, device="cuda", generator=g) < ignored, torch.full_like(spread, -100), spread)


def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split(",")]


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case=case)
    op = case["op"]
    if op == "ortho":
        s["x"] = _gradient(g, case["rows"], case["cols"], DT[case["dtype"]], pad=case["pad"])
        s["out"] = torch.empty(case["rows"], case["cols"], dtype=DT[case["out"]], device="cuda")
    elif op == "muon":
        s["items"] = []
        for r, k in _shapes(case):
            p = _normal(g, r, k, sigma=k**-0.5)
            grad = _gradient(g, r, k, DT[case["grad"]])
            m = _gradient(g, r, k, F32, 3e-4).reshape(-1)
            if case["momentum"] == "uf8":
                codes, top = _encode(m)
                s["items"].append(dict(p=p, g=grad, m=codes, meta=top, p1=torch.empty_like(p), m1=torch.empty_like(codes), meta1=torch.empty_like(top)))
            else:
                s["items"].append(dict(p=p, g=grad, m=m, p1=torch.empty_like(p), m1=torch.empty_like(m)))
    elif op == "xent":
        t, d, v = case["tokens"], case["hidden"], case["vocab"]
        w = _normal(g, v, d, sigma=0.02)
        target = _tokens(g, t, v) if t > 1 else _tokens(g, t, v, 0.0)
        h = _normal(g, t, d) + w[target.clamp_min(0)] * (6.0 / (0.02 * math.sqrt(d)))  # a model that has learnt something
        s.update(h=h.to(BF16), w=w.to(BF16), target=target, loss=torch.empty(t, device="cuda"), scale=1.0 / t)
        s["weight"] = torch.rand(t, device="cuda", generator=g) if case["weight"] else None
        s["dh"] = None if case["dh"] == "none" else torch.empty(t, d, dtype=DT[case["dh"]], device="cuda")
        s["dw"] = None if case["dw"] == "none" else torch.empty(v, d, dtype=DT[case["dw"]], device="cuda")
        s["base"] = _normal(g, v, d, sigma=1e-4).to(DT[case["dw"]]) if case["base"] else None
    elif op == "embed":
        s.update(table=_normal(g, case["vocab"], case["hidden"], sigma=0.02).to(DT[case["dtype"]]),
                 ids=_tokens(g, case["tokens"], case["vocab"], 0.02 if case["tokens"] > 1 else 0.0).to(getattr(torch, case["ids"])),
                 out=torch.empty(case["tokens"], case["hidden"], dtype=DT[case["out"]], device="cuda"), scale=math.sqrt(case["hidden"]))
    else:
        s.update(dy=_matrix(g, case["tokens"], case["hidden"], case["pad"], DT[case["dtype"]], 1e-3),
                 ids=_tokens(g, case["tokens"], case["vocab"]).to(getattr(torch, case["ids"])),
                 dw=torch.empty(case["vocab"], case["hidden"], dtype=DT[case["grad"]], device="cuda"), scale=math.sqrt(case["hidden"]))
        s["base"] = _normal(g, case["vocab"], case["hidden"], sigma=1e-4).to(s["dw"].dtype) if case["base"] else None
    return s


def _encode(m):
    """The 8-bit code of an fp32 vector: (signed bytes of whole blocks, largest magnitude of each block)."""
    n = m.numel()
    v = torch.zeros(-(-n // BLOCK) * BLOCK, dtype=F64, device=m.device)
    v[:n] = m
    v = v.view(-1, BLOCK)
    top = v.abs().amax(1, keepdim=True)
    codes = (v * (127.0 / top)).round().clamp(-127, 127)
    codes = torch.where(top > 0, codes, torch.zeros_like(codes))
    return codes.to(torch.int8).view(-1), top.float().view(-1)


def _decode(codes, top, n):
    """The fp32 values that a code stands for."""
    return (codes.double().view(-1, BLOCK) * (top.double() / 127.0)[:, None]).float().view(-1)[:n]


# ----------------------------------------------------------------------------------- plain forms
def _orthogonal(x):
    """The orthogonalised fp32 matrix."""
    a, b, c = COEFS
    x = x / (x.double().square().sum().sqrt() + EPS).float()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    for _ in range(STEPS):
        s = x @ x.t()
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.t() if tall else x


def _rms_scale(rows, cols):
    return 0.2 * math.sqrt(max(rows, cols))


def _plain_muon(case, i):
    n = i["p"].numel()
    m = _decode(i["m"], i["meta"], n) if "meta" in i else i["m"]
    g = i["g"].double().reshape(-1)
    m = (BETA * m.double() + (1.0 - BETA) * g).float()
    u = (BETA * m.double() + (1.0 - BETA) * g).float().view(i["p"].shape)
    p = i["p"] * (1.0 - case["lr"] * case["wd"]) - (case["lr"] * _rms_scale(*u.shape)) * _orthogonal(u)
    return dict(p=p, m=_decode(*_encode(m), n) if "meta" in i else m)


def _plain_xent(s):
    c = s["case"]
    inside = (s["target"] >= 0) & (s["target"] < c["vocab"])
    at = s["target"].clamp(0, c["vocab"] - 1)[:, None]
    h, w = s["h"].float(), s["w"].float()
    logits = h @ w.t()
    top = logits.amax(1, keepdim=True)
    lse = (logits - top).exp().sum(1, keepdim=True).log() + top
    out = dict(loss=torch.where(inside, (lse - logits.gather(1, at))[:, 0], 0.0))
    if c["dh"] == "none":
        return out
    d = (logits - lse).exp()
    d.scatter_add_(1, at, torch.full_like(lse, -1.0))
    d *= torch.where(inside, s["scale"] * (1.0 if s["weight"] is None else s["weight"]), 0.0)[:, None]
    dw = d.t() @ h
    dw = dw if s["base"] is None else dw + s["base"].float()
    return dict(out, dh=(d @ w).to(s["dh"].dtype), dw=dw.to(s["dw"].dtype))


def _plain(s):
    c = s["case"]
    if c["op"] == "ortho":
        return _orthogonal(s["x"].float()).to(s["out"].dtype)
    if c["op"] == "muon":
        return [_plain_muon(c, i) for i in s["items"]]
    if c["op"] == "xent":
        return _plain_xent(s)
    inside = (s["ids"] >= 0) & (s["ids"] < c["vocab"])
    at = s["ids"].clamp(0, c["vocab"] - 1)
    if c["op"] == "embed":
        return torch.where(inside[:, None], s["table"][at].float() * s["scale"], 0.0).to(s["out"].dtype)
    dy = torch.where(inside[:, None], s["dy"].float() * s["scale"], 0.0)
    dw = torch.zeros(c["vocab"], c["hidden"], device="cuda") if s["base"] is None else s["base"].float()
    return torch.index_add(dw, 0, at, dy).to(s["dw"].dtype)


# ------------------------------------------------------------------------- the framework's calls
def _own(s):
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import muon, vocab

    c = s["case"]
    op = c["op"]
    if op == "ortho":
        if "ws" not in s:
            s["ws"] = al.workspace(muon.orthogonalize_workspace_bytes(s["x"], s["out"]))
        muon.orthogonalize(s["x"], s["out"], s["ws"], steps=STEPS, coefs=COEFS, eps=EPS)
        return s["out"]
    if op == "muon":
        if "ws" not in s:
            s["states"] = [al.ParamState(i["p1"], i["g"], *i["p"].shape, m=i["m1"], m_meta=i.get("meta1")) for i in s["items"]]
            s["cfg"] = al.muon_cfg(lr=c["lr"], beta=BETA, weight_decay=c["wd"], eps=EPS, coefs=COEFS, steps=STEPS, parts=2, nesterov=True,
                                   scale=al.SCALE_RMS, grad_bf16=c["grad"] == "bf16", m=al.Spec(al.UF8 if c["momentum"] == "uf8" else al.FP32, BLOCK))
            s["arr"] = al.tensor_array(s["states"])
            s["ws"] = al.workspace(al.muon_workspace_bytes(s["states"], s["cfg"], arr=s["arr"]))
        # the step works in place: a pass begins from the parameters and momentum that it was given
        torch._foreach_copy_([i[k + "1"] for i in s["items"] for k in ("p", "m", "meta") if k in i],
                             [i[k] for i in s["items"] for k in ("p", "m", "meta") if k in i])
        al.muon_step(s["states"], s["cfg"], 1, s["ws"], arr=s["arr"])
        return [dict(p=i["p1"], m=_decode(i["m1"], i["meta1"], i["p"].numel()) if "meta" in i else i["m1"]) for i in s["items"]]
    if op == "xent":
        if "ws" not in s:
            s["ws"] = al.workspace(vocab.linear_xent_workspace_bytes(s["h"], s["w"], s["dh"], s["dw"]))
        vocab.linear_xent(s["h"], s["w"], s["target"], s["loss"], s["ws"], weight=s["weight"], scale=s["scale"], dh=s["dh"], dw=s["dw"],
                          base=s["base"])
        return {k: s[k] for k in ("loss", "dh", "dw") if s[k] is not None}
    if op == "embed":
        vocab.embed_forward(s["table"], s["ids"], s["out"], scale=s["scale"])
        return s["out"]
    if "ws" not in s:
        s["ws"] = al.workspace(vocab.embed_backward_workspace_bytes(s["dy"], s["dw"]))
    vocab.embed_backward(s["dy"], s["ids"], s["dw"], s["ws"], scale=s["scale"], base=s["base"])
    return s["dw"]


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------- work
def _size(kind):
    return 2 if kind == "bf16" else 4


def work(case):
    op = case["op"]
    if op == "ortho":
        n = case["rows"] * case["cols"]
        return dict(bytes=n * (_size(case["dtype"]) + _size(case["out"])), flops=_ns_flops(case["rows"], case["cols"]))
    if op == "muon":
        n = sum(r * k for r, k in _shapes(case))
        return dict(bytes=n * (8 + _size(case["grad"]) + (2 if case["momentum"] == "uf8" else 8)), flops=sum(_ns_flops(r, k) for r, k in _shapes(case)))
    t, d, v = case["tokens"], case["hidden"], case["vocab"]
    if op == "xent":
        grads = [k for k in ("dh", "dw") if case[k] != "none"]
        out = (t * d * _size(case["dh"]) + v * d * _size(case["dw"]) * (2 if case["base"] else 1)) if grads else 0
        return dict(bytes=2 * d * (t + v) + 12 * t + out, flops=2 * t * v * d * (1 + len(grads)))
    ids = t * (8 if case["ids"] == "int64" else 4)
    if op == "embed":
        return dict(bytes=t * d * (_size(case["dtype"]) + _size(case["out"])) + ids, flops=t * d)
    return dict(bytes=t * d * _size(case["dtype"]) + v * d * _size(case["grad"]) * (2 if case["base"] else 1) + ids, flops=2 * t * d)


# ------------------------------------------------------------------------------ 64-bit definitions
def _newton_schulz(u):
    a, b, c = COEFS
    y = u.double().contiguous()
    y = y / (torch.linalg.vector_norm(y) + EPS)
    if y.shape[0] > y.shape[1]:
        for _ in range(STEPS):
            k = torch.mm(y.t(), y)
            y = a * y + torch.mm(y, b * k + c * torch.mm(k, k))
    else:
        for _ in range(STEPS):
            k = torch.mm(y, y.t())
            y = a * y + torch.mm(b * k + c * torch.mm(k, k), y)
    return y


def _code_values(m, n):
    """What fp32 values stand for once they are coded: multiples of a 127th of their block's largest magnitude."""
    v = torch.nn.functional.pad(m.double(), (0, -n % BLOCK)).unflatten(0, (-1, BLOCK))
    most = v.abs().amax(1, keepdim=True)
    steps = torch.where(most > 0, v * (127.0 / most), torch.zeros_like(v)).round()
    return (steps * (most / 127.0)).flatten()[:n]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "ortho":
        return _newton_schulz(s["x"])
    if op == "muon":
        got = []
        for i in s["items"]:
            n = i["p"].numel()
            old = i["m"].double()
            if "meta" in i:
                old = (old.view(-1, BLOCK) * (i["meta"].double() / 127.0).unsqueeze(1)).flatten()[:n].to(F32).double()
            g = i["g"].double().flatten()
            m = torch.add(old * BETA, g, alpha=1.0 - BETA).to(F32)  # the momentum is an fp32 number by definition
            u = torch.add(m.double() * BETA, g, alpha=1.0 - BETA).view(i["p"].shape)
            step = case["lr"] * 0.2 * max(u.shape) ** 0.5
            got.append(dict(p=i["p"].double() * (1.0 - case["lr"] * case["wd"]) - step * _newton_schulz(u),
                            m=_code_values(m, n) if "meta" in i else m.double()))
        return got
    v = case["vocab"]
    if op == "xent":
        h, w = s["h"].double(), s["w"].double()
        keep = (s["target"] >= 0) & (s["target"] < v)
        z = torch.mm(h, w.t().contiguous())
        logp = z - torch.logsumexp(z, 1, keepdim=True)
        rows = torch.arange(z.shape[0], device="cuda")[keep]
        loss = torch.zeros(z.shape[0], dtype=F64, device="cuda")
        loss[keep] = -logp[rows, s["target"][keep]]
        if case["dh"] == "none":
            return dict(loss=loss)
        d = torch.exp(logp)
        d[rows, s["target"][keep]] -= 1.0
        share = s["scale"] * keep.double() * (1.0 if s["weight"] is None else s["weight"].double())
        d = d * share.unsqueeze(1)
        dw = torch.mm(d.t().contiguous(), h)
        return dict(loss=loss, dh=torch.mm(d, w), dw=dw if s["base"] is None else dw + s["base"].double())
    ids = s["ids"].long()
    keep = ((ids >= 0) & (ids < v)).nonzero().flatten()
    if op == "embed":
        y = torch.zeros(case["tokens"], case["hidden"], dtype=F64, device="cuda")
        y[keep] = s["table"].double()[ids[keep]] * s["scale"]
        return y
    order = keep[torch.argsort(ids[keep], stable=True)]
    sums = torch.zeros(v, case["hidden"], dtype=F64, device="cuda") if s["base"] is None else s["base"].double()
    return sums.index_put((ids[order],), s["dy"].double()[order] * s["scale"], accumulate=True)
