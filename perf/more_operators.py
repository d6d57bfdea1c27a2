"""Cases of the operators with which a model on a trained map is trained and
served whole: layer norm, the gated layer, the loss that takes what a teacher (the
map, or a larger model) and the labels say, and the product of matrices held in 8
bits.

``run`` computes them in elementary torch operations, in 32 bits and rounded
once at the end, or, where ``own`` is true, by the calls of
``paper_1905_09598_amd.local``.  ``exact`` gives the same outputs from the
definitions in 64 bits.

Sizes are those of the workload table and the benchmark (documents of 500 to
10,000 terms, maps of 100 to 10,000 units, 2048 floats) and of the paper's corpora
(637 x 4545); hidden widths and the longest rows of classes are generic.
"""
import math

import torch

own = False

DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
BLOCK = 128          # elements that share a scale where they are held in 8 bits
EPS = 1e-5


def listed():
    return [
        # One new document before it is answered: latency alone.
        {"name": "norm_serve_1x2048_bf16", "op": "norm", "dtype": "bf16", "n": 1, "width": 2048,
         "train": False, "beside": False},
        # A corpus of the paper's size, odd row length, single precision, trained.
        {"name": "norm_train_637x4545_fp32", "op": "norm", "dtype": "fp32", "n": 637,
         "width": 4545, "train": True, "beside": False},
        # The longest documents of the workload table, with the gradient of the path
        # that goes past the norm.
        {"name": "norm_train_20000x10000_fp16", "op": "norm", "dtype": "fp16", "n": 20000,
         "width": 10000, "train": True, "beside": True},
        # One document through a gated layer: one read of its matrices.
        {"name": "gated_serve_1x2048_8192_bf16", "op": "gated", "dtype": "bf16", "n": 1,
         "inner": 2048, "hidden": 8192, "act": "silu", "train": False},
        # A corpus of the workload table, hidden width off every tile.
        {"name": "gated_train_2000x2000_501_fp16", "op": "gated", "dtype": "fp16", "n": 2000,
         "inner": 2000, "hidden": 501, "act": "gelu", "train": True},
        # A training batch of the benchmark's rows.
        {"name": "gated_train_8192x2048_4096_bf16", "op": "gated", "dtype": "bf16", "n": 8192,
         "inner": 2048, "hidden": 4096, "act": "silu", "train": True},
        # The smallest workload: 200 documents on a map of 10 x 10 units, whose four
        # nearest units teach a gate; launches alone.
        {"name": "distill_200x100_top4_fp32", "op": "distill", "dtype": "fp32", "n": 200,
         "classes": 100, "k": 4, "temperature": 1.0, "rest": True, "label": False, "mix": 1.0,
         "closed": False},
        # A batch against the benchmark's map of 100 x 100 units: the teacher's eight
        # best, labels beside them, some documents without either.
        {"name": "distill_16001x10000_top8_bf16", "op": "distill", "dtype": "bf16", "n": 16001,
         "classes": 10000, "k": 8, "temperature": 2.0, "rest": True, "label": True, "mix": 0.7,
         "closed": True},
        # Rows longer than a workgroup holds, few of them.
        {"name": "distill_512x200003_top32_bf16", "op": "distill", "dtype": "bf16", "n": 512,
         "classes": 200003, "k": 32, "temperature": 1.5, "rest": False, "label": True,
         "mix": 0.5, "closed": False},
        # One new document against the benchmark's map, the gate held in 8 bits.
        {"name": "linear8_serve_1x2048_10000_bf16", "op": "linear8", "dtype": "bf16", "n": 1,
         "inner": 2048, "outer": 10000, "act": "none", "residual": False, "fresh": False},
        # A corpus of the paper's size through weights that are brought to 8 bits first;
        # rows that end within a block.
        {"name": "linear8_fresh_637x4545_501_fp16", "op": "linear8", "dtype": "fp16", "n": 637,
         "inner": 4545, "outer": 501, "act": "relu", "residual": False, "fresh": True},
        # A dense layer over a batch of documents, everything in its epilogue.
        {"name": "linear8_8192x2048_8192_bf16", "op": "linear8", "dtype": "bf16", "n": 8192,
         "inner": 2048, "outer": 8192, "act": "gelu", "residual": True, "fresh": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "gated", "distill", "linear8"])
    dtype = rng.choice(["bf16", "fp16", "fp32"])
    train = rng.random() < 0.6
    if op == "norm":
        width = _log(rng, 8, 20000)
        if rng.random() < 0.5:
            width = (width + 7) // 8 * 8
        return {"op": op, "dtype": dtype, "n": min(_log(rng, 1, 60000), 100000000 // width),
                "width": width, "train": train, "beside": train and rng.random() < 0.5}
    if op == "gated":
        while True:
            n, inner, hidden = _log(rng, 1, 40000), _log(rng, 64, 10000), _log(rng, 8, 8192)
            if rng.random() < 0.5:
                inner, hidden = (inner + 7) // 8 * 8, (hidden + 7) // 8 * 8
            flops = (12 if train else 4) * n * inner * hidden * (8 if dtype == "fp32" else 1)
            if flops <= 6e11:
                break
        return {"op": op, "dtype": dtype, "n": n, "inner": inner, "hidden": hidden,
                "act": rng.choice(["silu", "gelu", "none"]), "train": train}
    if op == "distill":
        classes = _log(rng, 4, 250000)
        label = rng.random() < 0.5
        return {"op": op, "dtype": dtype, "n": min(_log(rng, 1, 60000), 80000000 // classes or 1),
                "classes": classes, "k": rng.randint(1, min(32, classes)),
                "temperature": rng.choice([1.0, 1.5, 2.0, 4.0]), "rest": rng.random() < 0.5,
                "label": label, "mix": rng.choice([0.2, 0.5, 0.7]) if label else 1.0,
                "closed": rng.random() < 0.5}
    while True:
        n, inner, outer = _log(rng, 1, 40000), _log(rng, 64, 10000), _log(rng, 8, 10000)
        if 2 * n * inner * outer <= 3e11:
            break
    return {"op": op, "dtype": rng.choice(["bf16", "fp16"]), "n": n, "inner": inner,
            "outer": outer, "act": rng.choice(["none", "relu", "gelu", "silu"]),
            "residual": rng.random() < 0.5, "fresh": rng.random() < 0.5}


# ------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _documents(n, d, g):
    """Rows of Gaussian mixtures of 16 clusters, about unit variance a term."""
    centre = torch.randn(16, d, generator=g, device="cuda")
    which = torch.randint(0, 16, (n,), generator=g, device="cuda")
    return 0.8 * centre[which] + 0.6 * torch.randn(n, d, generator=g, device="cuda")


def prepare(case, seed):
    c, g = dict(case), _generator(seed)
    t = DTYPE[c["dtype"]]

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    s = {"case": c}
    if c["op"] == "norm":
        n, width = c["n"], c["width"]
        # rows of their own mean and scale
        s["x"] = (_documents(n, width, g) * (0.5 + rand(n, 1)) + 0.5 * randn(n, 1)).to(t)
        s["weight"] = (1 + 0.1 * randn(width)).to(t)
        s["bias"] = (0.1 * randn(width)).to(t)
        if c["train"]:
            s["dy"] = randn(n, width).to(t)
        s["beside"] = randn(n, width).to(t) if c["beside"] else None
    elif c["op"] == "gated":
        n, inner, hidden = c["n"], c["inner"], c["hidden"]
        s["x"] = _documents(n, inner, g).to(t)
        s["w"] = (randn(2, hidden, inner) / math.sqrt(inner)).to(t)
        s["bias"] = (0.1 * randn(2, hidden)).to(t)
        if c["train"]:
            s["dy"] = randn(n, hidden).to(t)
    elif c["op"] == "distill":
        n, classes, k = c["n"], c["classes"], c["k"]
        said = 2 * randn(n, classes)
        s["logits"] = (said + randn(n, classes)).to(t)     # a student some way on
        top = said.topk(k, dim=1)
        s["index"], s["teacher"] = top.indices.int(), top.values
        mass = (said / c["temperature"]).softmax(1).gather(1, top.indices).sum(1)
        s["rest"] = (1 - mass).clamp(min=0) if c["rest"] else None
        s["label"] = None
        if c["label"]:
            label = torch.where(rand(n) < 0.7, top.indices[:, 0],
                                torch.randint(0, classes, (n,), generator=g, device="cuda"))
            s["label"] = label.int()
        if c["closed"]:     # classes that are closed, choices and labels that are not there
            shut = rand(n, classes) < 0.05
            shut = shut.scatter(1, top.indices, False)
            if c["label"]:
                shut = shut.scatter(1, label.unsqueeze(1), False)
                s["label"][rand(n) < 0.05] = -1
            s["logits"][shut] = -math.inf
            s["index"][rand(n, k) < 0.1] = -1
            s["index"][rand(n) < 0.03] = -1
        s["dloss"] = (0.5 + rand(n)) / n
    else:
        n, inner, outer = c["n"], c["inner"], c["outer"]
        s["x"] = _documents(n, inner, g).to(t)
        w = (randn(outer, inner) / math.sqrt(inner)).to(t)
        if c["fresh"]:
            s["w"] = w
        else:               # as a served model holds it
            s["codes"], s["scale"] = _to_blocks(w)
        s["bias"] = (0.1 * randn(outer)).to(t)
        s["residual"] = randn(n, outer).to(t) if c["residual"] else None
    return s


# ------------------------------------------------------------- plain forms
def _act(z, kind):
    if kind == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if kind == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if kind == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, kind):
    if kind == "gelu":
        return (0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
                + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi)))
    if kind == "silu":
        q = 1 / (1 + torch.exp(-z))
        return q * (1 + z * (1 - q))
    return torch.ones_like(z)


def _plain_norm(s):
    c, t, x = s["case"], s["x"].dtype, s["x"].float()
    weight = s["weight"].float()
    off = x - x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt((off * off).mean(1, keepdim=True) + EPS)
    shown = off * rstd
    y = (shown * weight + s["bias"].float()).to(t)
    if not c["train"]:
        return {"y": y}
    dy = s["dy"].float()
    g = dy * weight
    dx = rstd * (g - g.mean(1, keepdim=True) - shown * (g * shown).mean(1, keepdim=True))
    if s["beside"] is not None:
        dx = dx + s["beside"].float()
    return {"y": y, "dx": dx.to(t), "dweight": (dy * shown).sum(0).to(t), "dbias": dy.sum(0).to(t)}


def _plain_gated(s):
    c, t, x = s["case"], s["x"].dtype, s["x"].float()
    hidden = c["hidden"]
    w = s["w"].float().view(2 * hidden, c["inner"])
    z = x @ w.t() + s["bias"].float().view(-1)
    gate, up = z[:, :hidden], z[:, hidden:]
    h = _act(gate, c["act"])
    y = (h * up).to(t)
    if not c["train"]:
        return {"y": y}
    dy = s["dy"].float()
    dz = torch.cat([dy * up * _act_slope(gate, c["act"]), dy * h], 1)
    return {"y": y, "dx": (dz @ w).to(t), "dw": (dz.t() @ x).view(2, hidden, -1).to(t),
            "dbias": dz.sum(0).view(2, hidden).to(t)}


def _plain_distill(s):
    c, x = s["case"], s["logits"].float()
    n, classes = x.shape
    heat, mix = c["temperature"], c["mix"]
    there = s["index"] >= 0
    at = torch.where(there, s["index"].long(), torch.full_like(s["index"], classes).long())
    inside = at.clamp(max=classes - 1)
    # the teacher: its choices that are there share what its rest leaves
    said = torch.where(there, s["teacher"] / heat, torch.full_like(s["teacher"], -math.inf))
    best = said.max(1, keepdim=True).values
    taught = best > -math.inf
    q = torch.exp(said - torch.where(taught, best, torch.zeros_like(best)))
    total = q.sum(1, keepdim=True)
    rest = s["rest"].unsqueeze(1) if s["rest"] is not None else torch.zeros_like(total)
    rest = torch.where(taught, rest, torch.zeros_like(rest))
    p = (1 - rest) * q / torch.where(taught, total, torch.ones_like(total))
    # the student
    a = x / heat
    top = a.max(1, keepdim=True).values
    e = torch.exp(a - top)
    z = e.sum(1, keepdim=True)
    chosen = torch.zeros(n, classes + 1, dtype=torch.bool, device=x.device)
    chosen = chosen.scatter(1, at, True)[:, :classes]
    others = torch.where(chosen, torch.zeros_like(e), e)
    zr = others.sum(1, keepdim=True)
    loga = a.gather(1, inside) - top - torch.log(z)
    zero = torch.zeros_like(p)
    soft = torch.where(p > 0, p * (torch.log(torch.where(p > 0, p, zero + 1)) - loga), zero).sum(1)
    left = torch.where(rest > 0, rest, torch.ones_like(rest))
    soft = soft + torch.where(rest > 0, left * (torch.log(left) - torch.log(zr / z)),
                              torch.zeros_like(rest)).squeeze(1)
    loss = mix * heat * heat * soft
    away = torch.where(rest > 0, 1 - rest * z / zr, torch.ones_like(rest))
    slope = torch.where(chosen, e / z, e / z * away)
    target = torch.zeros(n, classes + 1, device=x.device).scatter_add(1, at, p)[:, :classes]
    grad = torch.where(taught, mix * heat * (slope - target), torch.zeros_like(slope))
    if s["label"] is not None:
        known = (s["label"] >= 0).unsqueeze(1)
        which = s["label"].long().clamp(min=0).unsqueeze(1)
        top = x.max(1, keepdim=True).values
        e = torch.exp(x - top)
        z = e.sum(1, keepdim=True)
        hard = torch.log(z) + top - x.gather(1, which)
        hard = torch.where(known, hard, torch.zeros_like(hard))
        loss = loss + (1 - mix) * hard.squeeze(1)
        one = torch.zeros_like(x).scatter(1, which, 1.0)
        grad = grad + torch.where(known, (1 - mix) * (e / z - one), torch.zeros_like(one))
    return {"loss": loss, "dlogits": (grad * s["dloss"].unsqueeze(1)).to(s["logits"].dtype)}


def _to_blocks(x):
    """e4m3 codes, rows filled up with zeros to whole blocks, and each block's scale,
    the least power of two that brings its largest magnitude to 448 or below; the
    rows of scales are filled up to a multiple of four."""
    n, width = x.shape
    blocks = (width + BLOCK - 1) // BLOCK
    v = torch.nn.functional.pad(x.float(), (0, blocks * BLOCK - width)).view(n, blocks, BLOCK)
    size = v.abs()
    size = torch.where(size < math.inf, size, torch.zeros_like(size))
    m, e = torch.frexp(size.amax(2))
    e = torch.where(m > 0, e - 9 + (m > 0.875).int(), torch.full_like(e, -126)).clamp(min=-126)
    one = torch.ones_like(m)
    codes = (v * torch.ldexp(one, -e).unsqueeze(2)).to(torch.float8_e4m3fn)
    scale = torch.nn.functional.pad(torch.ldexp(one, e), (0, -blocks % 4), value=1.0)
    return codes.view(n, -1), scale.to(torch.float8_e8m0fnu)


def _from_blocks(codes, scale, width):
    blocks = codes.shape[1] // BLOCK
    v = codes.float().view(-1, blocks, BLOCK) * scale.float()[:, :blocks].unsqueeze(2)
    return v.view(-1, blocks * BLOCK)[:, :width]


def _plain_linear8(s):
    c, t = s["case"], s["x"].dtype
    out = {}
    codes, scale = _to_blocks(s["w"]) if c["fresh"] else (s["codes"], s["scale"])
    if c["fresh"]:
        out = {"codes": codes, "scale": scale}
    x = _from_blocks(*_to_blocks(s["x"]), c["inner"])
    y = _act(x @ _from_blocks(codes, scale, c["inner"]).t() + s["bias"].float(), c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out["y"] = y.to(t)
    return out


# ----------------------------------------------------- the framework's calls
def _own_norm(s):
    from paper_1905_09598_amd import local
    if not s["case"]["train"]:
        return {"y": local.norm(s["x"], s["weight"], s["bias"], EPS)}
    y, kept = local.norm(s["x"], s["weight"], s["bias"], EPS, keep=True)
    dx, dweight, dbias = local.norm_backward(s["dy"], s["x"], s["weight"], kept, s["beside"])
    return {"y": y, "dx": dx, "dweight": dweight, "dbias": dbias}


def _own_gated(s):
    from paper_1905_09598_amd import local
    c = s["case"]
    if not c["train"]:
        return {"y": local.gated(s["x"], s["w"], s["bias"], c["act"])}
    y, z = local.gated(s["x"], s["w"], s["bias"], c["act"], keep=True)
    dx, dw, dbias = local.gated_backward(s["dy"], s["x"], s["w"], z, c["act"])
    return {"y": y, "dx": dx, "dw": dw, "dbias": dbias}


def _own_distill(s):
    from paper_1905_09598_amd import local
    c = s["case"]
    loss, dlogits = local.distill(s["logits"], s["index"], s["teacher"], c["temperature"],
                                  s["rest"], s["label"], c["mix"], dloss=s["dloss"])
    return {"loss": loss, "dlogits": dlogits}


def _own_linear8(s):
    from paper_1905_09598_amd import local
    c = s["case"]
    if c["fresh"]:
        w = local.to_blocks(s["w"])
        y = local.linear8(s["x"], w, s["bias"], c["act"], s["residual"])
        return {"codes": w.codes, "scale": w.scale, "y": y}
    w = local.Blocks(s["codes"], s["scale"], c["inner"])
    return {"y": local.linear8(s["x"], w, s["bias"], c["act"], s["residual"])}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"norm": _own_norm, "gated": _own_gated, "distill": _own_distill,
                "linear8": _own_linear8}[op](state)
    return {"norm": _plain_norm, "gated": _plain_gated, "distill": _plain_distill,
            "linear8": _plain_linear8}[op](state)


def work(case):
    c, b = case, SIZE[case["dtype"]]
    if c["op"] == "norm":
        n, d = c["n"], c["width"]
        if not c["train"]:
            return {"bytes": (2 * n * d + 2 * d) * b, "flops": 8 * n * d}
        return {"bytes": ((5 if c["beside"] else 4) * n * d + 4 * d) * b, "flops": 20 * n * d}
    if c["op"] == "gated":
        n, i, h = c["n"], c["inner"], c["hidden"]
        once = n * i + 2 * h * i + 2 * h + n * h
        if not c["train"]:
            return {"bytes": once * b, "flops": 4 * n * i * h}
        return {"bytes": (once + n * h + n * i + 2 * h * i + 2 * h) * b, "flops": 12 * n * i * h}
    if c["op"] == "distill":
        n, v = c["n"], c["classes"]
        row = 8 * c["k"] + 8 + (4 if c["rest"] else 0) + (4 if c["label"] else 0)
        return {"bytes": 2 * n * v * b + n * row, "flops": (16 if c["label"] else 9) * n * v}
    n, i, o = c["n"], c["inner"], c["outer"]
    held = o * ((i + BLOCK - 1) // BLOCK) * (BLOCK + 1)
    bytes_ = (n * i + o + n * o * (2 if c["residual"] else 1)) * b + held
    return {"bytes": bytes_ + (o * i * b if c["fresh"] else 0), "flops": 2 * n * i * o}


# --------------------------------------------------- definitions in 64 bits
def _curve(z, kind):
    if kind == "relu":
        return z.clamp(min=0)
    if kind == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2))
    if kind == "silu":
        return z * torch.sigmoid(z)
    return z


def _grad(value, of, by):
    return torch.autograd.grad(value, of, by)


def _exact_norm(s):
    c = s["case"]
    x, w, b = (s[k].double().requires_grad_(c["train"]) for k in ("x", "weight", "bias"))
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    y = torch.addcmul(b, (x - mean) * torch.rsqrt(var + EPS), w)
    if not c["train"]:
        return {"y": y}
    dx, dw, db = _grad(y, (x, w, b), s["dy"].double())
    if s["beside"] is not None:
        dx = dx + s["beside"].double()
    return {"y": y.detach(), "dx": dx, "dweight": dw, "dbias": db}


def _exact_gated(s):
    c = s["case"]
    x, w, b = (s[k].double().requires_grad_(c["train"]) for k in ("x", "w", "bias"))
    y = _curve(x.mm(w[0].t()) + b[0], c["act"]) * (x.mm(w[1].t()) + b[1])
    if not c["train"]:
        return {"y": y}
    dx, dw, db = _grad(y, (x, w, b), s["dy"].double())
    return {"y": y.detach(), "dx": dx, "dw": dw, "dbias": db}


def _exact_distill(s):
    c = s["case"]
    x = s["logits"].double().requires_grad_()
    n, classes = x.shape
    heat = c["temperature"]
    there = s["index"] >= 0
    at = s["index"].long().clamp(min=0)
    said = (s["teacher"].double() / heat).masked_fill(~there, -math.inf)
    taught = there.any(1)
    logp = said.masked_fill(~taught.unsqueeze(1), 0.0).log_softmax(1)
    loga = (x / heat).log_softmax(1)
    rest = torch.zeros(n, dtype=torch.float64, device=x.device)
    if s["rest"] is not None:
        rest = s["rest"].double() * taught
    logp = logp + torch.log1p(-rest).unsqueeze(1)
    p = logp.exp() * there
    soft = (p * (logp.masked_fill(~there, 0.0) - loga.gather(1, at).masked_fill(~there, 0.0))).sum(1)
    if s["rest"] is not None:
        row = torch.arange(n, device=x.device).unsqueeze(1).expand_as(at)
        member = torch.zeros(n, classes, dtype=torch.bool, device=x.device)
        member[row[there], at[there]] = True
        others = loga.masked_fill(member, -math.inf)
        live = rest > 0
        logr = torch.where(live, rest, torch.ones_like(rest)).log()
        others = others.masked_fill(~live.unsqueeze(1), 0.0)   # rows without a rest: not used
        soft = soft + torch.where(live, rest * (logr - others.logsumexp(1)), torch.zeros_like(rest))
    loss = c["mix"] * heat * heat * soft
    if s["label"] is not None:
        known = s["label"] >= 0
        picked = x.log_softmax(1).gather(1, s["label"].long().clamp(min=0).unsqueeze(1)).squeeze(1)
        loss = loss - (1 - c["mix"]) * torch.where(known, picked, torch.zeros_like(picked))
    dx, = _grad(loss, (x,), s["dloss"].double())
    return {"loss": loss.detach(), "dlogits": dx}


def _shown(v):
    """v's values as 8 bits hold them, by rounding in 64 bits, with the exponents of
    their blocks' scales."""
    n, width = v.shape
    blocks = -(-width // BLOCK)
    full = torch.zeros(n, blocks * BLOCK, dtype=torch.float64, device=v.device)
    full[:, :width] = v.double()
    full = full.view(n, blocks, BLOCK)
    large = full.abs().amax(2)
    e = torch.ceil(torch.log2(large / 448)).clamp(min=-126)
    e = torch.where(large > 448 * torch.exp2(e), e + 1, e)
    e = torch.where(large <= 448 * torch.exp2(e - 1), e - 1, e).clamp(min=-126)
    u = full * torch.exp2(-e).unsqueeze(2)
    # 3 bits behind the leading one; below 2^-6 steps of 2^-9
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6))) - 3)
    held = torch.round(u / step) * step
    return held, e


def _exact_linear8(s):
    c = s["case"]

    def whole(held, e):
        return (held * torch.exp2(e).unsqueeze(2)).view(held.shape[0], -1)

    out = {}
    if c["fresh"]:
        held, e = _shown(s["w"])
        out["codes"] = held.reshape(held.shape[0], -1)
        out["scale"] = torch.nn.functional.pad(torch.exp2(e), (0, -e.shape[1] % 4), value=1.0)
        w = whole(held, e)
    else:
        blocks = s["codes"].shape[1] // BLOCK
        w = whole(s["codes"].double().view(-1, blocks, BLOCK),
                  torch.log2(s["scale"].double()[:, :blocks]))
    x = whole(*_shown(s["x"]))
    y = _curve(torch.addmm(s["bias"].double(), x, w.t()), c["act"])
    out["y"] = y if s["residual"] is None else y + s["residual"].double()
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "gated": _exact_gated, "distill": _exact_distill,
            "linear8": _exact_linear8}[s["case"]["op"]](s)
