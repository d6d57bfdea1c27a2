"""Cases of the operators that put local models on a trained map: the product
with its epilogue (a gate's scores, a dense layer), the routing of documents to
experts, the routed experts' products and the optimizer step over all their
tensors.

``run`` computes them in elementary torch operations, in 32 bits and rounded
once at the end, or, where ``own`` is true, by the calls of
``paper_1905_09598_amd.local``.  ``exact`` gives the same outputs from the
definitions in 64 bits.

Sizes are those of the workload table and the benchmark (documents of 500 to
10,000 terms, maps of 100 to 10,000 units, up to 100,000 samples of 2048
floats) and of the paper's corpora (637 x 4545); hidden widths are generic.
"""
import math

import torch

own = False

DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
BLOCK = 256          # elements that share a scale where states are held in 8 bits
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01


def listed():
    return [
        # One new document against the benchmark's map of 100 x 100 units: the
        # gate's scores, one read of the prototypes.
        {"name": "linear_serve_1x2048_10000_bf16", "op": "linear", "dtype": "bf16", "n": 1,
         "inner": 2048, "outer": 10000, "act": "none", "residual": False, "train": False},
        # A corpus of the paper's size on its map of 11 x 11 units, single
        # precision, odd row length: the gate trained with the experts.
        {"name": "linear_train_637x4545_121_fp32", "op": "linear", "dtype": "fp32", "n": 637,
         "inner": 4545, "outer": 121, "act": "none", "residual": False, "train": True},
        # A dense layer over a batch of documents, everything in its epilogue.
        {"name": "linear_8192x2048_8192_bf16", "op": "linear", "dtype": "bf16", "n": 8192,
         "inner": 2048, "outer": 8192, "act": "gelu", "residual": True, "train": False},
        # The same layer kind trained, other 16-bit type, an odd batch.
        {"name": "linear_train_16001x2048_2048_fp16", "op": "linear", "dtype": "fp16", "n": 16001,
         "inner": 2048, "outer": 2048, "act": "silu", "residual": True, "train": True},
        # One document routed while serving: latency alone.
        {"name": "route_serve_1x64_top2", "op": "route", "dtype": "bf16", "n": 1, "experts": 64,
         "k": 2, "mode": "softmax", "bias": False, "groups": 1, "top_groups": 1,
         "group_best": 1, "renormalise": True, "train": False, "empty": False},
        # A corpus on a map of 20 x 20 units, four units to a document; some
        # documents are empty and their rows are masked.
        {"name": "route_train_20000x400_top4", "op": "route", "dtype": "fp32", "n": 20000,
         "experts": 400, "k": 4, "mode": "softmax", "bias": False, "groups": 1, "top_groups": 1,
         "group_best": 1, "renormalise": False, "train": True, "empty": True},
        # Many experts in groups with a bias for balance, a large batch.
        {"name": "route_train_65536x256_top8_groups", "op": "route", "dtype": "bf16", "n": 65536,
         "experts": 256, "k": 8, "mode": "sigmoid", "bias": True, "groups": 8, "top_groups": 4,
         "group_best": 2, "renormalise": True, "train": True, "empty": False},
        # One document answered by the local models of its four units.
        {"name": "experts_serve_1x2048_1024_e64_top4", "op": "experts", "dtype": "bf16", "n": 1,
         "inner": 2048, "hidden": 1024, "experts": 64, "k": 4, "act": "gelu", "residual": True,
         "skew": 1.0, "train": False},
        # Training on a corpus of the workload table, a few documents to an
        # expert, sizes off every tile.
        {"name": "experts_train_2000x2000_501_e100_top2", "op": "experts", "dtype": "fp16",
         "n": 2000, "inner": 2000, "hidden": 501, "experts": 100, "k": 2, "act": "relu",
         "residual": False, "skew": 0.5, "train": True},
        # Training on the benchmark's rows, popular experts beside rare ones.
        {"name": "experts_train_8192x2048_1024_e16_top2", "op": "experts", "dtype": "bf16",
         "n": 8192, "inner": 2048, "hidden": 1024, "experts": 16, "k": 2, "act": "gelu",
         "residual": True, "skew": 0.5, "train": True},
        # The optimizer over a small gate and its experts: launches alone.
        {"name": "adamw_12x_small_fp32", "op": "adamw", "dtype": "fp32", "grad": "fp32",
         "tensors": 12, "total": 150000, "bits": 32, "master": False},
        # The optimizer over large experts in half precision, states in 8 bits.
        {"name": "adamw_18x_67M_bf16_8bit", "op": "adamw", "dtype": "bf16", "grad": "bf16",
         "tensors": 18, "total": 67000000, "bits": 8, "master": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "route", "experts", "adamw"])
    dtype = rng.choice(["bf16", "fp16", "fp32"])
    train = rng.random() < 0.5
    if op == "linear":
        while True:
            n, inner, outer = _log(rng, 1, 40000), _log(rng, 64, 10000), _log(rng, 8, 10000)
            if rng.random() < 0.5:
                inner, outer = (inner + 7) // 8 * 8, (outer + 7) // 8 * 8
            flops = (6 if train else 2) * n * inner * outer * (8 if dtype == "fp32" else 1)
            if flops <= 3.5e11:
                break
        return {"op": op, "dtype": dtype, "n": n, "inner": inner, "outer": outer,
                "act": rng.choice(["none", "relu", "gelu", "silu"]),
                "residual": rng.random() < 0.5, "train": train}
    if op == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        experts = groups * _log(rng, max(2, 4 // groups), 2048 // groups)
        n = min(_log(rng, 1, 60000), 12000000 // experts)
        top_groups = rng.randint(1, groups)
        k = rng.randint(1, min(8, top_groups * (experts // groups)))
        return {"op": op, "dtype": dtype, "n": n, "experts": experts, "k": k,
                "mode": rng.choice(["softmax", "sigmoid"]), "bias": rng.random() < 0.5,
                "groups": groups, "top_groups": top_groups, "group_best": rng.choice([1, 2]),
                "renormalise": rng.random() < 0.5, "train": train, "empty": rng.random() < 0.5}
    if op == "experts":
        while True:
            n, inner, hidden = _log(rng, 1, 20000), _log(rng, 64, 4000), _log(rng, 32, 2048)
            if rng.random() < 0.5:
                inner, hidden = (inner + 7) // 8 * 8, (hidden + 7) // 8 * 8
            experts, k = _log(rng, 4, 128), rng.randint(1, 4)
            flops = (12 if train else 4) * n * k * inner * hidden * (8 if dtype == "fp32" else 1)
            if flops <= 3e11 and experts * inner * hidden <= 1.3e8:
                break
        return {"op": op, "dtype": dtype, "n": n, "inner": inner, "hidden": hidden,
                "experts": experts, "k": k, "act": rng.choice(["relu", "gelu", "silu"]),
                "residual": rng.random() < 0.5, "skew": rng.choice([0.0, 0.5, 1.0]),
                "train": train}
    return {"op": op, "dtype": dtype, "grad": rng.choice([dtype, "fp32"]),
            "tensors": rng.randint(1, 20), "total": _log(rng, 3000, 30000000),
            "bits": rng.choice([8, 32]), "master": dtype != "fp32" and rng.random() < 0.5}


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


def _popularity(experts, skew, g):
    """What a gate's scores have in common for all documents: a few experts
    are asked for often."""
    rank = torch.randperm(experts, generator=g, device="cuda") + 1
    return -skew * torch.log(rank.float())


def _sizes(c):
    """Element counts of the optimizer's tensors: matrices of falling size
    and short bias vectors between them, odd counts among them."""
    t, total = c["tensors"], c["total"]
    share = [1.0 / (1 + i // 2) if i % 2 == 0 else 0.002 for i in range(t)]
    return [max(1, int(total * s / sum(share)) - (i % 3)) for i, s in enumerate(share)]


def _padded(sizes):
    return [(s + BLOCK - 1) // BLOCK * BLOCK for s in sizes]


def prepare(case, seed):
    c, g = dict(case), _generator(seed)
    t = DTYPE[c["dtype"]]

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    s = {"case": c}
    if c["op"] == "linear":
        n, inner, outer = c["n"], c["inner"], c["outer"]
        s["x"] = _documents(n, inner, g).to(t)
        s["w"] = (randn(outer, inner) / math.sqrt(inner)).to(t)
        s["bias"] = (0.1 * randn(outer)).to(t)
        s["residual"] = randn(n, outer).to(t) if c["residual"] else None
        if c["train"]:
            s["dy"] = randn(n, outer).to(t)
    elif c["op"] == "route":
        n, experts = c["n"], c["experts"]
        scores = randn(n, experts) + _popularity(experts, 0.3, g)
        if c["empty"]:      # documents without a term, and experts closed to some documents
            scores[torch.rand(n, experts, generator=g, device="cuda") < 0.1] = -math.inf
            scores[torch.rand(n, generator=g, device="cuda") < 0.02] = -math.inf
        s["scores"] = scores.to(t)
        s["bias"] = 0.05 * randn(experts) if c["bias"] else None
        if c["train"]:
            s["dweight"] = randn(n, c["k"])
    elif c["op"] == "experts":
        n, inner, hidden, experts = c["n"], c["inner"], c["hidden"], c["experts"]
        s["x"] = _documents(n, inner, g).to(t)
        s["w1"] = (randn(experts, hidden, inner) / math.sqrt(inner)).to(t)
        s["b1"] = (0.1 * randn(experts, hidden)).to(t)
        s["w2"] = (randn(experts, inner, hidden) / math.sqrt(hidden)).to(t)
        s["b2"] = (0.1 * randn(experts, inner)).to(t)
        scores = randn(n, experts) + _popularity(experts, c["skew"], g)
        top = scores.topk(c["k"], dim=1)
        s["index"], s["weight"] = top.indices.int(), top.values.softmax(1)
        s["residual"] = randn(n, inner).to(t) if c["residual"] else None
        if c["train"]:
            s["dy"] = randn(n, inner).to(t)
    else:
        sizes = _sizes(c)
        room = sum(_padded(sizes))
        s["params"] = [(0.05 * randn(z)).to(t) for z in sizes]
        s["grads"] = [(1e-3 * randn(z)).to(DTYPE[c["grad"]]) for z in sizes]
        # the states of a run some steps old, each tensor from a multiple of BLOCK on
        mean, square = torch.zeros(room, device="cuda"), torch.zeros(room, device="cuda")
        at = 0
        for z, p in zip(sizes, _padded(sizes)):
            mean[at:at + z] = 3e-4 * randn(z)
            square[at:at + z] = 1e-8 * (0.1 + randn(z).square())
            at += p
        if c["bits"] == 8:
            s["mean"], s["mean_scale"] = _to_blocks(mean)
            s["square"], s["square_scale"] = _to_blocks(square.sqrt())
        else:
            s["mean"], s["square"] = mean, square
        s["master"] = (torch.cat([torch.nn.functional.pad(p.float(), (0, q - p.numel()))
                                  for p, q in zip(s["params"], _padded(sizes))])
                       if c["master"] else None)
        s["step"] = 20
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
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "gelu":
        return (0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
                + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi)))
    if kind == "silu":
        q = 1 / (1 + torch.exp(-z))
        return q * (1 + z * (1 - q))
    return torch.ones_like(z)


def _plain_linear(s):
    c, t = s["case"], s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t() + s["bias"].float()
    y = _act(z, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    if not c["train"]:
        return {"y": y.to(t)}
    dz = s["dy"].float()
    if c["act"] != "none":
        dz = dz * _act_slope(z, c["act"])
    return {"y": y.to(t), "dx": (dz @ w).to(t), "dw": (dz.t() @ x).to(t),
            "dbias": dz.sum(0).to(t)}


def _plain_order(index, experts):
    """Slots (document * k + choice) by expert, their order kept; the first
    slot of each expert; absent slots (-1) last, as -1."""
    flat = index.reshape(-1).long()
    key = torch.where(flat < 0, torch.full_like(flat, experts), flat)
    order = torch.sort(key, stable=True).indices
    count = torch.zeros(experts + 1, dtype=torch.long, device=flat.device)
    count.index_add_(0, key, torch.ones_like(key))
    offsets = torch.cat([torch.zeros_like(count[:1]), count[:experts].cumsum(0)])
    there = torch.arange(flat.numel(), device=flat.device) < offsets[experts]
    return offsets, torch.where(there, order, torch.full_like(order, -1))


def _plain_route(s):
    c, x = s["case"], s["scores"].float()
    n, experts, k, groups = x.shape[0], c["experts"], c["k"], c["groups"]
    softmax = c["mode"] == "softmax"
    p = x if softmax else 1 / (1 + torch.exp(-x))
    pick = p if s["bias"] is None else p + s["bias"]
    pick = torch.where(x > -math.inf, pick, torch.full_like(pick, -math.inf))
    if groups > 1:
        best = pick.view(n, groups, -1).sort(dim=2, descending=True).values[:, :, :c["group_best"]]
        none = best == -math.inf
        value = torch.where(none, torch.zeros_like(best), best).sum(2)
        value = torch.where(none[:, :, 0], torch.full_like(value, -math.inf), value)
        first = value.sort(dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        stays = torch.zeros(n, groups, dtype=torch.bool, device=x.device).scatter(1, first, True)
        stays = stays.unsqueeze(2).expand(-1, -1, experts // groups).reshape(n, experts)
        pick = torch.where(stays, pick, torch.full_like(pick, -math.inf))
    top = pick.sort(dim=1, descending=True, stable=True)
    value, at = top.values[:, :k], top.indices[:, :k]
    here = value > -math.inf
    index = torch.where(here, at, torch.full_like(at, -1)).int()
    zero = torch.zeros_like(value)
    low = x.max(1, keepdim=True).values
    low = torch.where(low > -math.inf, low, torch.zeros_like(low))
    chosen = x.gather(1, at)
    if softmax:
        e = torch.exp(x - low)
        total = e.sum(1, keepdim=True)
        every = e / torch.where(total > 0, total, torch.ones_like(total))
        if c["renormalise"]:
            top1 = torch.where(here, chosen, torch.full_like(chosen, -math.inf)).max(
                1, keepdim=True).values
            top1 = torch.where(top1 > -math.inf, top1, torch.zeros_like(top1))
            q = torch.where(here, torch.exp(chosen - top1), zero)
            total = q.sum(1, keepdim=True)
            weight = q / torch.where(total > 0, total, torch.ones_like(total))
        else:
            weight = torch.where(here, every.gather(1, at), zero)
    else:
        q = torch.where(here, p.gather(1, at), zero)
        total = q.sum(1, keepdim=True)
        total = torch.where(total > 0, total, torch.ones_like(total))
        weight = q / total if c["renormalise"] else q
    offsets, order = _plain_order(index, experts)
    out = {"index": index, "weight": weight, "offsets": offsets.int(), "order": order.int()}
    if c["train"]:
        g = torch.where(here, s["dweight"], zero)
        if softmax and not c["renormalise"]:
            mean = (g * weight).sum(1, keepdim=True)
            full = torch.zeros_like(x).scatter(1, at, g)
            out["dscores"] = (every * (full - mean)).to(s["scores"].dtype)
        else:
            if c["renormalise"]:
                g = g - (g * weight).sum(1, keepdim=True)
            d = weight * g if softmax else q * (1 - q) * g / (total if c["renormalise"] else 1)
            out["dscores"] = torch.zeros_like(x).scatter(1, at, d).to(s["scores"].dtype)
    return out


def _plain_experts(s):
    c, t = s["case"], s["x"].dtype
    x, index, weight = s["x"].float(), s["index"].long(), s["weight"]
    n, k = index.shape
    w1, b1, w2, b2 = (s[name] for name in ("w1", "b1", "w2", "b2"))
    if not c["train"] and n * k <= c["experts"]:  # fewer slots than experts: their matrices alone
        z = (w1[index].float() @ x[:, None, :, None]).squeeze(3) + b1[index].float()
        h = _act(z, c["act"])
        y = (w2[index].float() @ h.unsqueeze(3)).squeeze(3) + b2[index].float()
        out = (weight.unsqueeze(2) * y).sum(1)
        if s["residual"] is not None:
            out = out + s["residual"].float()
        return {"y": out.to(t)}
    # every expert's rows side by side, filled up with zeros to the longest
    flat = index.reshape(-1)
    offsets, order = _plain_order(index, c["experts"])
    longest = int((offsets[1:] - offsets[:-1]).max())
    of = flat[order]
    place = torch.empty_like(order)
    place[order] = of * longest + torch.arange(n * k, device=x.device) - offsets[of]
    row = torch.arange(n, device=x.device).repeat_interleave(k)

    def spread(v):
        full = torch.zeros(c["experts"] * longest, v.shape[1], device=v.device)
        full[place] = v
        return full.view(c["experts"], longest, -1)

    def back(v):
        return v.reshape(c["experts"] * longest, -1)[place]

    xs, w1, w2 = spread(x[row]), w1.float(), w2.float()
    z = torch.bmm(xs, w1.transpose(1, 2).contiguous()) + b1.float().unsqueeze(1)
    h = _act(z, c["act"])
    y = back(torch.bmm(h, w2.transpose(1, 2).contiguous()) + b2.float().unsqueeze(1))
    out = (weight.unsqueeze(2) * y.view(n, k, -1)).sum(1)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    if not c["train"]:
        return {"y": out.to(t)}
    dy = s["dy"].float()
    dweight = (dy.unsqueeze(1) * y.view(n, k, -1)).sum(2)
    ds = spread(weight.reshape(-1, 1) * dy[row])
    dw2 = torch.bmm(ds.transpose(1, 2).contiguous(), h)
    dz = torch.bmm(ds, w2) * _act_slope(z, c["act"])
    dw1 = torch.bmm(dz.transpose(1, 2).contiguous(), xs)
    dx = back(torch.bmm(dz, w1)).view(n, k, -1).sum(1)
    return {"y": out.to(t), "dx": dx.to(t), "dweight": dweight.to(t), "dw1": dw1.to(t),
            "db1": dz.sum(1).to(t), "dw2": dw2.to(t), "db2": ds.sum(1).to(t)}


def _to_blocks(v):
    """e4m3 values and a scale for each block: its largest magnitude is 448."""
    b = v.view(-1, BLOCK)
    top = b.abs().amax(1, keepdim=True).clamp(min=1e-30)
    q = (b * (448.0 / top)).to(torch.float8_e4m3fn)
    return q.view(-1), (top / 448.0).view(-1)


def _from_blocks(q, scale):
    return (q.float().view(-1, BLOCK) * scale.unsqueeze(1)).view(-1)


def _plain_adamw(s):
    c = s["case"]
    s["step"] += 1
    step, eight = s["step"], c["bits"] == 8
    sizes = [p.numel() for p in s["params"]]
    pads = _padded(sizes)

    def flat(tensors):
        return torch.cat([torch.nn.functional.pad(v.float(), (0, q - v.numel()))
                          for v, q in zip(tensors, pads)])

    g = flat(s["grads"])
    p = s["master"] if c["master"] else flat(s["params"])
    if eight:
        m = _from_blocks(s["mean"], s["mean_scale"])
        r = _from_blocks(s["square"], s["square_scale"])
        v = r * r
    else:
        m, v = s["mean"], s["square"]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    root = torch.sqrt(v)
    p = p * (1 - LR * DECAY) - (m * (LR / (1 - BETA1 ** step))) / (
        root * (1 / math.sqrt(1 - BETA2 ** step)) + EPS)
    if eight:
        q, scale = _to_blocks(m)
        s["mean"].copy_(q)
        s["mean_scale"].copy_(scale)
        q, scale = _to_blocks(root)
        least = torch.full_like(p, 2.0 ** -9).to(torch.float8_e4m3fn)
        s["square"].copy_(torch.where((q.float() == 0) & (root > 0), least.float(), q.float()))
        s["square_scale"].copy_(scale)
    else:
        s["mean"].copy_(m)
        s["square"].copy_(v)
    if c["master"]:
        s["master"].copy_(p)
    parts = torch.split(p, pads)
    torch._foreach_copy_(s["params"], [v[:z] for v, z in zip(parts, sizes)])
    return _adamw_outputs(s)


def _adamw_outputs(s):
    names = ("params", "mean", "square", "mean_scale", "square_scale", "master")
    return {k: s[k] for k in names if s.get(k) is not None}


# ----------------------------------------------------- the framework's calls
def _own_linear(s):
    from paper_1905_09598_amd import local
    c = s["case"]
    if not c["train"]:
        return {"y": local.linear(s["x"], s["w"], s["bias"], c["act"], s["residual"])}
    y, z = local.linear(s["x"], s["w"], s["bias"], c["act"], s["residual"], keep=True)
    dx, dw, dbias = local.linear_backward(s["dy"], s["x"], s["w"], z, c["act"])
    return {"y": y, "dx": dx, "dw": dw, "dbias": dbias}


def _own_route(s):
    from paper_1905_09598_amd import local
    c = s["case"]
    r = local.route(s["scores"], c["k"], s["bias"], c["mode"], c["groups"], c["top_groups"],
                    c["group_best"], c["renormalise"])
    out = {"index": r.index, "weight": r.weight, "offsets": r.offsets, "order": r.order}
    if c["train"]:
        out["dscores"] = local.route_backward(s["dweight"], s["scores"], r)
    return out


def _own_experts(s):
    from paper_1905_09598_amd import local
    c = s["case"]
    r = local.dispatch(s["index"], s["weight"], c["experts"])
    w = (s["w1"], s["b1"], s["w2"], s["b2"])
    if not c["train"]:
        return {"y": local.experts(s["x"], r, *w, c["act"], s["residual"])}
    y, kept = local.experts(s["x"], r, *w, c["act"], s["residual"], keep=True)
    d = local.experts_backward(s["dy"], s["x"], r, *w, kept, c["act"])
    return {"y": y, "dx": d.x, "dweight": d.weight, "dw1": d.w1, "db1": d.b1, "dw2": d.w2,
            "db2": d.b2}


def _own_adamw(s):
    from paper_1905_09598_amd import local
    if "optimizer" not in s:     # made once, as a training program does
        states = {k: s[k] for k in ("mean", "square", "mean_scale", "square_scale", "master")
                  if s.get(k) is not None}
        s["optimizer"] = local.AdamW(s["params"], lr=LR, betas=(BETA1, BETA2), eps=EPS,
                                     weight_decay=DECAY, bits=s["case"]["bits"],
                                     step=s["step"], state=states)
    s["optimizer"].step(s["grads"])
    return _adamw_outputs(s)


def run(state):
    op = state["case"]["op"]
    if own:
        return {"linear": _own_linear, "route": _own_route, "experts": _own_experts,
                "adamw": _own_adamw}[op](state)
    return {"linear": _plain_linear, "route": _plain_route, "experts": _plain_experts,
            "adamw": _plain_adamw}[op](state)


def work(case):
    c, b = case, SIZE[case["dtype"]]
    if c["op"] == "linear":
        n, i, o = c["n"], c["inner"], c["outer"]
        once = n * i + o * i + o + n * o * (2 if c["residual"] else 1)
        if not c["train"]:
            return {"bytes": once * b, "flops": 2 * n * i * o}
        return {"bytes": (once + n * o + n * i + o * i + o) * b, "flops": 6 * n * i * o}
    if c["op"] == "route":
        n, e, k = c["n"], c["experts"], c["k"]
        bytes_ = n * e * b + n * k * 12 + (e + 1) * 4 + (e * 4 if c["bias"] else 0)
        if c["train"]:
            bytes_ += n * k * 4 + n * e * b
        return {"bytes": bytes_, "flops": n * e * (10 if c["train"] else 5)}
    if c["op"] == "experts":
        n, i, h, e, k = c["n"], c["inner"], c["hidden"], c["experts"], c["k"]
        used = e if c["train"] else min(e, n * k)
        weights = used * (2 * i * h + i + h)
        once = weights + n * i * (3 if c["residual"] else 2)
        flops = 4 * n * k * i * h
        if not c["train"]:
            return {"bytes": once * b + n * k * 8, "flops": flops}
        return {"bytes": (once + weights + 2 * n * i) * b + n * k * 12, "flops": 3 * flops}
    total = sum(_sizes(c))
    state = 16 if c["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": total * (2 * b + SIZE[c["grad"]] + state + (8 if c["master"] else 0)
                              - (b if c["master"] else 0)), "flops": 15 * total}


# --------------------------------------------------- definitions in 64 bits
def _curve(z, kind):
    """An activation and its slope."""
    if kind == "relu":
        return z.clamp(min=0), (z > 0).double()
    if kind == "gelu":
        below = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * below, below + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "silu":
        q = torch.sigmoid(z)
        return z * q, q + z * q * (1 - q)
    return z, torch.ones_like(z)


def _exact_linear(s):
    c = s["case"]
    x, w = s["x"].double(), s["w"].double()
    z = torch.addmm(s["bias"].double(), x, w.t())
    y, slope = _curve(z, c["act"])
    out = {"y": y if s["residual"] is None else y + s["residual"].double()}
    if c["train"]:
        dz = s["dy"].double() * slope
        out.update(dx=dz.mm(w), dw=dz.t().mm(x), dbias=dz.sum(0))
    return out


def _exact_route(s):
    c, x = s["case"], s["scores"].double()
    n, experts, k, groups = x.shape[0], c["experts"], c["k"], c["groups"]
    per = experts // groups
    softmax = c["mode"] == "softmax"
    pick = x.clone() if softmax else torch.sigmoid(x)
    if s["bias"] is not None:
        pick += s["bias"].double()
    pick[x == -math.inf] = -math.inf
    rows = torch.arange(n, device=x.device)
    if groups > 1:
        value = torch.empty(n, groups, dtype=torch.float64, device=x.device)
        for j in range(groups):
            part = pick[:, j * per:(j + 1) * per].topk(min(c["group_best"], per), 1).values
            value[:, j] = part.masked_fill(part == -math.inf, 0).sum(1)
            value[part[:, 0] == -math.inf, j] = -math.inf
        open_ = torch.zeros(n, groups, dtype=torch.bool, device=x.device)
        for _ in range(c["top_groups"]):
            j = value.argmax(1)
            open_[rows, j] = True
            value[rows, j] = -math.inf
        for j in range(groups):
            pick[~open_[:, j], j * per:(j + 1) * per] = -math.inf
    chosen = torch.zeros(n, experts, dtype=torch.float64, device=x.device)
    index = torch.empty(n, k, dtype=torch.long, device=x.device)
    there = torch.empty(n, k, dtype=torch.bool, device=x.device)
    for j in range(k):
        value, index[:, j] = pick.max(1)
        there[:, j] = value > -math.inf
        chosen[rows, index[:, j]] = torch.maximum(chosen[rows, index[:, j]], there[:, j].double())
        pick[rows, index[:, j]] = -math.inf
    if softmax:
        shown = x.masked_fill(chosen == 0, -math.inf) if c["renormalise"] else x
        p = torch.softmax(shown, 1).nan_to_num(0.0)
    else:
        p = torch.sigmoid(x)
        p[x == -math.inf] = 0
    total = torch.ones(n, 1, dtype=torch.float64, device=x.device)
    if c["renormalise"] and not softmax:
        total = (p * chosen).sum(1, keepdim=True)
        total[total == 0] = 1
    weight = (p / total).gather(1, index) * there
    out = {"index": None, "weight": weight, "offsets": None, "order": None}
    if c["train"]:
        g = torch.zeros_like(x).scatter_add(1, index, s["dweight"].double() * there)
        if softmax:
            out["dscores"] = p * (g - (p * g).sum(1, keepdim=True))
        else:
            if c["renormalise"]:
                g = (g - (g * chosen * p / total).sum(1, keepdim=True)) * chosen
            out["dscores"] = g * p * (1 - p) / total
    return out


def _exact_experts(s):
    c = s["case"]
    x, index, weight = s["x"].double(), s["index"].long(), s["weight"].double()
    n, k = index.shape
    y = torch.zeros(n, c["inner"], dtype=torch.float64, device=x.device)
    if s["residual"] is not None:
        y += s["residual"].double()
    names = ("w1", "b1", "w2", "b2")
    out = {}
    if c["train"]:
        dy, dx, dweight = s["dy"].double(), torch.zeros_like(x), torch.zeros_like(weight)
        out = {"d" + v: torch.zeros_like(s[v], dtype=torch.float64) for v in names}
    for e in range(c["experts"]):
        row, choice = (index == e).nonzero(as_tuple=True)
        if not row.numel():
            continue
        w1, b1, w2, b2 = (s[v][e].double() for v in names)
        xe, ge = x[row], weight[row, choice].unsqueeze(1)
        z = xe.mm(w1.t()) + b1
        h, slope = _curve(z, c["act"])
        ye = h.mm(w2.t()) + b2
        y.index_add_(0, row, ge * ye)
        if c["train"]:
            dweight[row, choice] = (dy[row] * ye).sum(1)
            de = ge * dy[row]
            out["dw2"][e], out["db2"][e] = de.t().mm(h), de.sum(0)
            dz = de.mm(w2) * slope
            out["dw1"][e], out["db1"][e] = dz.t().mm(xe), dz.sum(0)
            dx.index_add_(0, row, dz.mm(w1))
    out["y"] = y
    if c["train"]:
        out.update(dx=dx, dweight=dweight)
    return out


def _exact_adamw(s):
    c, step = s["case"], s["step"] + 1
    eight = c["bits"] == 8

    def held(name):
        v = s[name].double()
        if eight:
            v = (v.view(-1, BLOCK) * s[name + "_scale"].double().unsqueeze(1)).view(-1)
        return v * v if eight and name == "square" else v

    mean, square = held("mean"), held("square")
    params, at = [], 0
    m_new, v_new = torch.zeros_like(mean), torch.zeros_like(square)
    master = torch.zeros_like(mean)
    for p, g in zip(s["params"], s["grads"]):
        z = p.numel()
        here = slice(at, at + z)
        g = g.double()
        m_new[here] = BETA1 * mean[here] + (1 - BETA1) * g
        v_new[here] = BETA2 * square[here] + (1 - BETA2) * g * g
        p = s["master"][here].double() if c["master"] else p.double()
        m_hat, v_hat = m_new[here] / (1 - BETA1 ** step), v_new[here] / (1 - BETA2 ** step)
        p = p - LR * DECAY * p - LR * m_hat / (v_hat.sqrt() + EPS)
        params.append(p)
        master[here] = p
        at += (z + BLOCK - 1) // BLOCK * BLOCK
    out = {"params": params}
    if eight:       # what is held is a rounding; the scales have a value
        out.update(mean=None, square=None,
                   mean_scale=m_new.view(-1, BLOCK).abs().amax(1).clamp(min=1e-30) / 448,
                   square_scale=v_new.sqrt().view(-1, BLOCK).amax(1).clamp(min=1e-30) / 448)
    else:
        out.update(mean=m_new, square=v_new)
    if c["master"]:
        out["master"] = master
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "route": _exact_route, "experts": _exact_experts,
            "adamw": _exact_adamw}[s["case"]["op"]](s)
