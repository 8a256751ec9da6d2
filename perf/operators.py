"""Training with activations held in 8 bits, as cases that can be timed and compared.

The operators: the activation code (save and load), layer and RMS norm with their backward pass, the gated
activation of a transformer's MLP with its backward pass from saved codes, and the weight gradient of a linear layer
whose input was saved in 8 bits. Widths are those of the repository's 1.1B and 7B lists (2048 / 5632 / 256 and
4096 / 11008), its 1024 x 1024 matrix and its odd test widths (500, 1001, 1750, 2731); token counts run from one
token to a batch of four sequences of 2048.

An activation code holds a matrix row by row in blocks of 32, 64 or 128 columns: a signed byte per value and one
exponent byte E per block. E is the biased fp32 exponent of the block's largest magnitude less 6 (at least 1), a value
is coded as the nearest multiple of 2^(E - 127), clamped to 127 steps, and a block that holds a NaN or an infinity has
E = 255 and decodes to NaN.
"""
from __future__ import annotations

import math

import torch

own = False

F32, BF16 = torch.float32, torch.bfloat16
DT = {"fp32": F32, "bf16": BF16}


# ------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the MLP's hidden activation of a 7B-wide layer, four sequences of 2048: the largest tensor a layer keeps
        dict(name="code-8192x11008", op="code", rows=8192, cols=11008, pad=0, dtype="bf16", block=64),
        # an odd-width fp32 activation that is a slice of a wider buffer
        dict(name="code-odd-1500x1001", op="code", rows=1500, cols=1001, pad=6, dtype="fp32", block=128),
        # one token's norm when a model answers: latency is all there is
        dict(name="norm-1x4096", op="norm", kind="rms", rows=1, cols=4096, pad=0, dtype="bf16", save=False, block=64),
        # the pre-norm of a 7B-wide layer in training, its output's normalised form saved in 8 bits
        dict(name="norm-save-8192x4096", op="norm", kind="rms", rows=8192, cols=4096, pad=0, dtype="bf16", save=True, block=64),
        # layer norm of a small model of odd width, fp32
        dict(name="norm-layer-4096x1750", op="norm", kind="layer", rows=4096, cols=1750, pad=0, dtype="fp32", save=False, block=64),
        # the backward pass of the pre-norm from the 8-bit code, the residual's gradient added
        dict(name="dnorm-code-8192x4096", op="dnorm", kind="rms", rows=8192, cols=4096, pad=0, dtype="bf16", grad="bf16",
             code=True, add=True, block=64),
        # layer norm's backward pass from its input, weight and bias gradients in fp32, odd width
        dict(name="dnorm-layer-2048x1750", op="dnorm", kind="layer", rows=2048, cols=1750, pad=0, dtype="fp32", grad="fp32",
             code=False, add=False, block=64),
        # the gated activation of the 1.1B model, one sequence of 2048, gate and up saved
        dict(name="swiglu-2048x5632", op="swiglu", rows=2048, cols=5632, pad=0, dtype="bf16", save=True, block=64),
        # its backward pass at the 7B widths, with the code of the recomputed output for the next weight gradient
        dict(name="dswiglu-8192x11008", op="dswiglu", rows=8192, cols=11008, pad=0, dtype="bf16", save=True, block=64),
        # weight gradient of the 1024 x 1024 matrix over a short microbatch, fp32 gradients
        dict(name="wgrad-512-1024x1024", op="wgrad", rows=512, out=1024, cols=1024, pad=0, dtype="bf16", grad="fp32", block=64,
             scale=False, base=False, bias=False),
        # the gate matrix of a 7B-wide layer, behind its norm: the largest weight gradient of a step
        dict(name="wgrad-8192-11008x4096", op="wgrad", rows=8192, out=11008, cols=4096, pad=0, dtype="bf16", grad="bf16",
             block=64, scale=True, base=False, bias=False),
        # a key projection of the 1.1B model over a ragged batch, added to what earlier microbatches left, with the
        # gradient of a bias: few outputs, a long sum
        dict(name="wgrad-6001-256x2048", op="wgrad", rows=6001, out=256, cols=2048, pad=0, dtype="bf16", grad="fp32", block=32,
             scale=True, base=True, bias=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    n = _log_uniform(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.6 else n  # most models round their widths


def draw(rng):
    op = rng.choice(["code", "norm", "dnorm", "swiglu", "dswiglu", "wgrad", "wgrad"])
    c = dict(op=op, rows=_log_uniform(rng, 1, 16384), cols=_width(rng, 40, 11008), pad=rng.choice([0, 0, 0, 8, 5]),
             dtype=rng.choice(["bf16", "bf16", "bf16", "fp32"]), block=rng.choice([32, 64, 64, 128]))
    if op == "wgrad":
        c.update(out=_width(rng, 40, 11008), grad=rng.choice(["bf16", "fp32"]), scale=rng.random() < 0.5,
                 base=rng.random() < 0.5, bias=rng.random() < 0.3)
        while c["rows"] * c["cols"] * c["out"] * (3 if c["dtype"] == "fp32" else 1) > 8192 * 4096 * 11008:
            c["rows"] = c["rows"] // 2 + 1
        return c
    while c["rows"] * c["cols"] * (2 if c["dtype"] == "fp32" else 1) > (8192 * 4096 if "norm" in op else 8192 * 11008):
        c["rows"] = c["rows"] // 2 + 1
    if "norm" in op:
        c["kind"] = rng.choice(["layer", "rms"])
    if op in ("norm", "swiglu", "dswiglu"):
        c["save"] = rng.random() < 0.6
    if op == "dnorm":
        c.update(grad=rng.choice(["bf16", "fp32"]), code=rng.random() < 0.6, add=rng.random() < 0.6)
    return c


# ----------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _matrix(g, rows, cols, pad, dtype, sigma=1.0, spread=0.0, shift=0.0, dead=False):
    """rows x cols of a buffer of cols + pad columns: normal values, channels whose sizes spread log-normally by
    `spread` (some run far hotter than the rest, as in a transformer), one row in 64 all zero where `dead` (padding tokens)."""
    x = torch.empty(rows, cols + pad, dtype=F32, device="cuda").normal_(0.0, sigma, generator=g)
    if spread:
        x *= torch.empty(cols + pad, dtype=F32, device="cuda").normal_(0.0, spread, generator=g).exp_()
    x += shift
    if dead:
        x *= torch.rand(rows, 1, device="cuda", generator=g) >= 1 / 64
    return x.to(dtype)[:, :cols]


def _like(rows, cols, pad, dtype):
    return torch.empty(rows, cols + pad, dtype=dtype, device="cuda")[:, :cols]


def _encode(x, block):
    """(codes, exponents) of a matrix: codes int8 [rows, blocks * block], exponents uint8 [rows, blocks]."""
    rows, cols = x.shape
    nb = -(-cols // block)
    v = torch.zeros(rows, nb * block, dtype=F32, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, nb, block)
    top = v.abs().amax(-1, keepdim=True).view(torch.int32) >> 23
    e = torch.where(top == 255, top, (top - 6).clamp_min(1))
    inverse = ((254 - e).clamp_min(0) << 23).view(F32)
    codes = (v * inverse).round().clamp(-127, 127)
    codes = torch.where(e == 255, torch.zeros_like(codes), codes)
    return codes.to(torch.int8).view(rows, nb * block), e.to(torch.uint8).view(rows, nb)


def _decode(codes, exps, cols, block):
    """The fp32 values that a matrix's codes stand for (all of them bf16 numbers)."""
    scale = (exps.to(torch.int32) << 23).view(F32)
    return (codes.view(exps.shape[0], exps.shape[1], block).to(F32) * scale[:, :, None]).view(codes.shape)[:, :cols]


def prepare(case, seed):
    g = _gen(seed)
    op, rows, cols, pad, block, dt = (case[k] for k in ("op", "rows", "cols", "pad", "block", "dtype"))
    dt = DT[dt]
    nb = -(-cols // block)
    s = dict(case=case)

    def buffers():  # where a call writes codes
        return (torch.zeros(rows, nb * block, dtype=torch.int8, device="cuda"),
                torch.zeros(rows, nb, dtype=torch.uint8, device="cuda"))

    if op == "code":
        s.update(x=_matrix(g, rows, cols, pad, dt, spread=0.8, dead=True), code=buffers(), out=_like(rows, cols, pad, dt))
    elif op == "norm":
        layer = case["kind"] == "layer"
        s.update(x=_matrix(g, rows, cols, pad, dt, spread=0.4, shift=0.1), gamma=_vector(g, cols, 1.0), y=_like(rows, cols, pad, dt),
                 rstd=torch.empty(rows, device="cuda"), eps=1e-5)
        s["beta"] = _vector(g, cols, 0.0) if layer else None
        s["mean"] = torch.empty(rows, device="cuda") if layer else None
        if case["save"]:
            s.update(code=buffers(), loaded=_like(rows, cols, 0, BF16))
    elif op == "dnorm":
        x = _matrix(g, rows, cols, pad, dt, spread=0.4, shift=0.1)
        mean = x.float().mean(1) if case["kind"] == "layer" else None
        d = x.float() if mean is None else x.float() - mean[:, None]
        rstd = (d.square().mean(1) + 1e-5).rsqrt()
        s.update(dy=_matrix(g, rows, cols, pad, dt, 1e-3, dead=True), gamma=_vector(g, cols, 1.0), mean=mean, rstd=rstd)
        s["add"] = _matrix(g, rows, cols, pad, dt, 1e-3) if case["add"] else None
        if case["code"]:
            s["code"] = _encode(d * rstd[:, None], block)
        else:
            s["x"] = x
        s.update(dx=_like(rows, cols, pad, dt), dgamma=torch.empty(cols, dtype=DT[case["grad"]], device="cuda"))
        s["dbeta"] = torch.empty_like(s["dgamma"]) if case["kind"] == "layer" else None
    elif op == "swiglu":
        s.update(gate=_matrix(g, rows, cols, pad, dt, 1.5, spread=0.5), up=_matrix(g, rows, cols, pad, dt, spread=0.5),
                 h=_like(rows, cols, pad, dt))
        if case["save"]:
            s.update(codes=[buffers(), buffers()], loaded=[_like(rows, cols, 0, BF16), _like(rows, cols, 0, BF16)])
    elif op == "dswiglu":
        s.update(dh=_matrix(g, rows, cols, pad, dt, 1e-3, dead=True),
                 codes=[_encode(_matrix(g, rows, cols, 0, F32, 1.5, spread=0.2), block),
                        _encode(_matrix(g, rows, cols, 0, F32, spread=0.2), block)],
                 dgate=_like(rows, cols, pad, dt), dup=_like(rows, cols, pad, dt))
        if case["save"]:
            s.update(code=buffers(), loaded=_like(rows, cols, 0, BF16))
    else:
        gt = DT[case["grad"]]
        s.update(dy=_matrix(g, rows, case["out"], pad, dt, 1e-3, dead=True),
                 code=_encode(_matrix(g, rows, cols, 0, F32, spread=0.5), block),
                 dw=torch.empty(case["out"], cols, dtype=gt, device="cuda"))
        s["gamma"] = _vector(g, cols, 1.0) if case["scale"] else None
        s["beta"] = _vector(g, cols, 0.0) if case["scale"] and case["bias"] else None
        s["base"] = _matrix(g, case["out"], cols, 0, gt, 1e-2) if case["base"] else None
        s["dbias"] = torch.empty(case["out"], dtype=gt, device="cuda") if case["bias"] else None
    return s


def _vector(g, n, center):
    return center + torch.empty(n, dtype=F32, device="cuda").normal_(0.0, 0.1, generator=g)


# ----------------------------------------------------------------------------------- plain forms
def _sigmoid(x):
    return 1 / (1 + (-x).exp())


def _loaded(x, block):
    """What a matrix is after it was saved and loaded again."""
    return _decode(*_encode(x, block), x.shape[1], block).to(BF16)


def _plain(s):
    c = s["case"]
    op, cols, block, dt = c["op"], c["cols"], c["block"], DT[c["dtype"]]
    if op == "code":
        return _decode(*_encode(s["x"].float(), block), cols, block).to(dt)
    if op == "norm":
        x = s["x"].float()
        mean = x.mean(1) if c["kind"] == "layer" else None
        d = x if mean is None else x - mean[:, None]
        rstd = 1 / (d.square().mean(1) + s["eps"]).sqrt()
        xh = d * rstd[:, None]
        y = xh * s["gamma"]
        y = y if s["beta"] is None else y + s["beta"]
        out = dict(y=y.to(dt), rstd=rstd)
        if mean is not None:
            out["mean"] = mean
        if c["save"]:
            out["saved"] = _loaded(xh, block)
        return out
    if op == "dnorm":
        dy = s["dy"].float()
        if c["code"]:
            xh = _decode(*s["code"], cols, block)
        else:
            xh = (s["x"].float() if s["mean"] is None else s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        a = dy * s["gamma"]
        v = a - xh * (a * xh).mean(1, keepdim=True)
        if c["kind"] == "layer":
            v = v - a.mean(1, keepdim=True)
        dx = s["rstd"][:, None] * v
        dx = dx if s["add"] is None else dx + s["add"].float()
        gt = DT[c["grad"]]
        out = dict(dx=dx.to(dt), dgamma=(dy * xh).sum(0).to(gt))
        if c["kind"] == "layer":
            out["dbeta"] = dy.sum(0).to(gt)
        return out
    if op == "swiglu":
        gate, up = s["gate"].float(), s["up"].float()
        out = dict(h=(gate * _sigmoid(gate) * up).to(dt))
        if c["save"]:
            out.update(gate=_loaded(gate, block), up=_loaded(up, block))
        return out
    if op == "dswiglu":
        gate, up = (_decode(*k, cols, block) for k in s["codes"])
        dh, sg = s["dh"].float(), _sigmoid(gate)
        out = dict(dgate=(dh * up * sg * (1 + gate * (1 - sg))).to(dt), dup=(dh * gate * sg).to(dt))
        if c["save"]:
            out["saved"] = _loaded(gate * sg * up, block)
        return out
    dy, gt = s["dy"].float(), DT[c["grad"]]
    dw = dy.t() @ _decode(*s["code"], cols, block)
    total = dy.sum(0) if c["bias"] else None
    dw = dw if s["gamma"] is None else dw * s["gamma"]
    dw = dw if s["beta"] is None else dw + total[:, None] * s["beta"]
    dw = dw if s["base"] is None else dw + s["base"].float()
    return dict(dw=dw.to(gt), **(dict(dbias=total.to(gt)) if c["bias"] else {}))


# ------------------------------------------------------------------------- the framework's calls
def _own(s):
    import paper_2608_22322_amd as al
    from paper_2608_22322_amd import activations as act

    c = s["case"]
    op, cols, block = c["op"], c["cols"], c["block"]

    def code(pair):
        return act.ActCode(pair[0], pair[1], c["rows"], cols, block)

    if "own" not in s:  # what a program sets up once: handles of its code buffers, workspaces
        s["own"] = {k: code(s[k]) for k in ("code",) if k in s}
        s["own"]["codes"] = [code(p) for p in s.get("codes", ())]
        kind = {"rms": act.RMS, "layer": act.LAYER}.get(c.get("kind"))
        if op == "dnorm":
            s["own"]["ws"] = al.workspace(act.norm_backward_workspace_bytes(kind, c["rows"], cols, dtype=DT[c["dtype"]]))
        elif op == "wgrad":
            s["own"]["ws"] = al.workspace(act.linear_wgrad_workspace_bytes(s["dy"], s["own"]["code"], s["dw"]))
        s["own"]["kind"] = kind
    o = s["own"]
    if op == "code":
        act.quantize(s["x"], o["code"])
        act.dequantize(o["code"], s["out"])
        return s["out"]
    if op == "norm":
        saved = o.get("code")
        act.norm_forward(o["kind"], s["x"], s["y"], s["mean"], s["rstd"], gamma=s["gamma"], beta=s["beta"], eps=s["eps"], code=saved)
        out = dict(y=s["y"], rstd=s["rstd"])
        if c["kind"] == "layer":
            out["mean"] = s["mean"]
        if saved is not None:
            act.dequantize(saved, s["loaded"])
            out["saved"] = s["loaded"]
        return out
    if op == "dnorm":
        act.norm_backward(o["kind"], s["dy"], o["code"] if c["code"] else s["x"], s["mean"], s["rstd"], s["dx"], gamma=s["gamma"],
                          dgamma=s["dgamma"], dbeta=s["dbeta"], add=s["add"], ws=o["ws"])
        out = dict(dx=s["dx"], dgamma=s["dgamma"])
        if s["dbeta"] is not None:
            out["dbeta"] = s["dbeta"]
        return out
    if op == "swiglu":
        if not c["save"]:
            act.swiglu_forward(s["gate"], s["up"], s["h"])
            return dict(h=s["h"])
        act.swiglu_forward(s["gate"], s["up"], s["h"], *o["codes"])
        act.dequantize(o["codes"][0], s["loaded"][0])
        act.dequantize(o["codes"][1], s["loaded"][1])
        return dict(h=s["h"], gate=s["loaded"][0], up=s["loaded"][1])
    if op == "dswiglu":
        act.swiglu_backward(s["dh"], *o["codes"], s["dgate"], s["dup"], h_code=o.get("code"))
        out = dict(dgate=s["dgate"], dup=s["dup"])
        if c["save"]:
            act.dequantize(o["code"], s["loaded"])
            out["saved"] = s["loaded"]
        return out
    act.linear_wgrad(s["dy"], o["code"], s["dw"], o["ws"], gamma=s["gamma"], beta=s["beta"], base=s["base"], dbias=s["dbias"])
    return dict(dw=s["dw"], **(dict(dbias=s["dbias"]) if c["bias"] else {}))


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------- work
def work(case):
    rows, cols, block = case["rows"], case["cols"], case["block"]
    n, w = rows * cols, 2 if case["dtype"] == "bf16" else 4
    coded = rows * (-(-cols // block)) * (block + 1)  # codes and exponents of one matrix
    op = case["op"]
    if op == "code":
        return dict(bytes=2 * n * w, flops=4 * n)
    if op == "norm":
        return dict(bytes=2 * n * w + 4 * cols + 4 * rows + (2 * n if case["save"] else 0), flops=8 * n)
    if op == "dnorm":
        return dict(bytes=2 * n * w + (coded if case["code"] else n * w) + (n * w if case["add"] else 0) + 8 * cols + 4 * rows, flops=12 * n)
    if op == "swiglu":
        return dict(bytes=3 * n * w + (4 * n if case["save"] else 0), flops=8 * n)
    if op == "dswiglu":
        return dict(bytes=3 * n * w + 2 * coded + (2 * n if case["save"] else 0), flops=16 * n)
    gw = 2 if case["grad"] == "bf16" else 4
    m = case["out"]
    return dict(bytes=rows * m * w + coded + m * cols * gw * (2 if case["base"] else 1), flops=2 * rows * m * cols)


# ------------------------------------------------------------------------------ 64-bit definitions
def _nearest(x, block):
    """Save and load in binary64: the step of a block is 2^(floor(log2 max) - 6), never under 2^-126."""
    rows, cols = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -cols % block)).unflatten(1, (-1, block))
    most = v.abs().amax(-1, keepdim=True)
    step = torch.exp2(torch.clamp(torch.frexp(most).exponent.double() - 7, min=-126.0))
    return ((v / step).round().clamp(-127, 127) * step).flatten(1)[:, :cols]


def _values(pair, cols, block):
    codes, exps = pair
    return (codes.double().unflatten(1, (-1, block)) * torch.exp2(exps.double() - 127).unsqueeze(-1)).flatten(1)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    op, cols, block = case["op"], case["cols"], case["block"]
    if op == "code":
        return _nearest(s["x"], block)
    if op == "norm":
        x = s["x"].double()
        layer = case["kind"] == "layer"
        mu = x.sum(1, keepdim=True) / cols if layer else torch.zeros(x.shape[0], 1, dtype=torch.float64, device="cuda")
        r = ((x - mu).pow(2).sum(1, keepdim=True) / cols + s["eps"]).pow(-0.5)
        xh = (x - mu) * r
        y = xh * s["gamma"].double() + (s["beta"].double() if layer else 0.0)
        return dict(y=y, rstd=r[:, 0], **(dict(mean=mu[:, 0]) if layer else {}), **(dict(saved=_nearest(xh, block)) if case["save"] else {}))
    if op == "dnorm":
        r, dy = s["rstd"].double()[:, None], s["dy"].double()
        layer = case["kind"] == "layer"
        mu = s["mean"].double()[:, None] if layer else 0.0
        xh = _values(s["code"], cols, block) if case["code"] else (s["x"].double() - mu) * r
        a = dy * s["gamma"].double()
        dx = a - xh * ((a * xh).sum(1, keepdim=True) / cols)
        if layer:
            dx = dx - a.sum(1, keepdim=True) / cols
        dx = dx * r + (0.0 if s["add"] is None else s["add"].double())
        return dict(dx=dx, dgamma=(dy * xh).sum(0), **(dict(dbeta=dy.sum(0)) if layer else {}))
    if op == "swiglu":
        gate, up = s["gate"].double(), s["up"].double()
        h = gate * torch.sigmoid(gate) * up
        return dict(h=h, **(dict(gate=_nearest(gate, block), up=_nearest(up, block)) if case["save"] else {}))
    if op == "dswiglu":
        gate, up = (_values(k, cols, block) for k in s["codes"])
        dh, p = s["dh"].double(), torch.sigmoid(gate)
        return dict(dgate=dh * up * (p + gate * p * (1 - p)), dup=dh * gate * p,
                    **(dict(saved=_nearest(gate * p * up, block)) if case["save"] else {}))
    dy = s["dy"].double()
    dw = torch.mm(dy.t().contiguous(), _values(s["code"], cols, block).contiguous())
    if s["gamma"] is not None:
        dw *= s["gamma"].double()
    if s["beta"] is not None:
        dw += torch.outer(dy.sum(0), s["beta"].double())
    if s["base"] is not None:
        dw += s["base"].double()
    return dict(dw=dw, **(dict(dbias=dy.sum(0)) if case["bias"] else {}))
