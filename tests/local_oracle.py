"""The local models' operators in 64 bits on the CPU, from their definitions
(no test functions here), and the bounds their kernels are held to.

Bounds.  u is the unit roundoff of an element type (bf16 2^-8, fp16 2^-11, fp32
2^-24) with half a least subnormal beside it, v = 2^-24 that of the sums.  A sum
of K products in any order is off by at most (K + 8) v times the sum of their
magnitudes (the 8 for the epilogue's few operations and the transcendental
functions' last places); a stored value by u of itself; a value that passes
through an intermediate held in 16 bits by u of that on the way.
"""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
V = 2.0 ** -24
# largest magnitudes of the activations' first and second derivatives
SLOPE = {"none": 1.0, "relu": 1.0, "gelu": 1.13, "silu": 1.1}
BEND = {"none": 0.0, "relu": 0.0, "gelu": 0.8, "silu": 0.5}


def d(t):
    return None if t is None else t.detach().double().cpu()


def act(z, kind):
    if kind == "relu":
        return z.clamp(min=0)
    if kind == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2))
    if kind == "silu":
        return z * torch.sigmoid(z)
    return z


def act_slope(z, kind):
    if kind == "relu":
        return (z > 0).double()
    if kind == "gelu":
        return (0.5 * torch.special.erfc(-z / math.sqrt(2))
                + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
    if kind == "silu":
        q = torch.sigmoid(z)
        return q * (1 + z * (1 - q))
    return torch.ones_like(z)


def stored(value, dtype):
    """Bound of one rounding to dtype."""
    return U[dtype] * value.abs() + TINY[dtype]


def linear(x, w, b, kind, r, dtype):
    """((y, bound), (z, bound)) of a product with its epilogue."""
    z = x @ w.t() + (0 if b is None else b)
    size = x.abs() @ w.abs().t() + (0 if b is None else b.abs())
    zerr = (x.shape[1] + 8) * V * size
    y = act(z, kind)
    yerr = SLOPE[kind] * zerr + 8 * V * z.abs()
    if r is not None:
        y = y + r
        yerr = yerr + 4 * V * r.abs()
    return (y, yerr + stored(y, dtype)), (z, zerr + stored(z, dtype))


def linear_backward(dy, x, w, z, zerr, kind, dtype, dyerr=None, rounded=None):
    """{"dx", "dw", "db"}: (value, bound); dyerr: bound of dy's own error; rounded:
    whether dz is held in dtype (by default where there is an activation)."""
    s = act_slope(z, kind)
    dz = dy * s
    err = dy.abs() * (BEND[kind] * zerr + 16 * V)
    if kind == "relu":      # next to the kink either slope is right
        err = err + dy.abs() * (z.abs() <= zerr).double()
    if dyerr is not None:
        err = err + dyerr * SLOPE[kind]
    if kind != "none" if rounded is None else rounded:
        err = err + stored(dz, dtype)
    n, out = dz.shape
    dx, dw, db = dz @ w, dz.t() @ x, dz.sum(0)
    full = dz.abs() + err
    return {"dx": (dx, err @ w.abs() + (out + 8) * V * (full @ w.abs()) + stored(dx, dtype)),
            "dw": (dw, err.t() @ x.abs() + (n + 8) * V * (full.t() @ x.abs())
                   + stored(dw, dtype)),
            "db": (db, err.sum(0) + (n + 8) * V * full.sum(0) + stored(db, dtype))}


def close(got, want, what=""):
    """Every element of the kernel's result within its bound (1 % on top for the
    bounds' own second-order terms)."""
    value, bound = want
    got = d(got)
    assert got.shape == value.shape, (what, got.shape, value.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(value)), what
    off = ((got - value).abs() - 1.01 * bound).nan_to_num(0.0)
    if off.numel():
        at = int(off.argmax())
        assert off.flatten()[at] <= 0, (
            what, at, float(got.flatten()[at]), float(value.flatten()[at]),
            float(bound.flatten()[at]))


# ------------------------------------------------------------------ routing
def route(scores, k, bias=None, gate="softmax", groups=1, top_groups=1, group_best=1,
          renormalise=True, scale=1.0):
    """(index, weight) from the definition, row by row, the choice by values in
    32 bits as the kernel holds them (ties and near ties have one answer)."""
    n, experts = scores.shape
    index = torch.full((n, k), -1, dtype=torch.int64)
    weight = torch.zeros(n, k, dtype=torch.float64)
    per = experts // groups
    s32 = scores.float()
    v32 = s32 if gate == "softmax" else 1 / (1 + torch.exp(-s32))
    if bias is not None:
        v32 = v32 + bias.float()
    for i in range(n):
        s = scores[i].double()
        if torch.isnan(s).any() or (gate == "softmax" and (s == math.inf).any()):
            weight[i] = math.nan
            continue
        v = {e: float(v32[i, e]) for e in range(experts)
             if s[e] > -math.inf and v32[i, e] > -math.inf}
        if groups > 1:
            value = {}
            for g in range(groups):
                best = sorted((v[e] for e in range(g * per, (g + 1) * per) if e in v),
                              reverse=True)[:group_best]
                if best:
                    value[g] = float(torch.tensor(best, dtype=torch.float32).sum())
            stay = sorted(value, key=lambda g: (-value[g], g))[:top_groups]
            v = {e: x for e, x in v.items() if e // per in stay}
        chosen = sorted(v, key=lambda e: (-v[e], e))[:k]
        if not chosen:
            continue
        index[i, :len(chosen)] = torch.tensor(chosen)
        if gate == "softmax":
            p = torch.softmax(s[chosen] if renormalise else s, 0)
            p = p if renormalise else p[chosen]
        else:
            p = torch.sigmoid(s[chosen])
            if renormalise:
                p = p / p.sum() if p.sum() > 0 else torch.zeros_like(p)
        weight[i, :len(chosen)] = scale * p
    return index, weight


def route_weight(scores, index, gate, renormalise, scale):
    """Weights of given choices, differentiable in the scores (64 bits)."""
    here = index >= 0
    at = index.clamp(min=0)
    low = scores.detach().amax(1, keepdim=True)
    e = torch.exp(scores - torch.where(low > -math.inf, low, torch.zeros_like(low)))
    p = e if gate == "softmax" else torch.sigmoid(scores)
    q = torch.where(here, p.gather(1, at), torch.zeros_like(p[:, :1]))
    if renormalise:
        total = q.sum(1, keepdim=True)
    else:
        total = e.sum(1, keepdim=True) if gate == "softmax" else torch.ones_like(q[:, :1])
    return scale * q / torch.where(total > 0, total, torch.ones_like(total))


# ------------------------------------------------------------------ experts
def experts(x, index, weight, w1, b1, w2, b2, kind, residual):
    """The joined answers, differentiable (64 bits)."""
    y = torch.zeros(x.shape[0], (w1 if w2 is None else w2).shape[1], dtype=torch.float64)
    if residual is not None:
        y = y + residual
    for i in range(index.shape[0]):
        for j in range(index.shape[1]):
            e = int(index[i, j])
            if e < 0:
                continue
            a = w1[e] @ x[i] + (0 if b1 is None else b1[e])
            if w2 is not None:
                a = w2[e] @ act(a, kind) + (0 if b2 is None else b2[e])
            y = y.index_add(0, torch.tensor([i]), (weight[i, j] * a).unsqueeze(0))
    return y


# ---------------------------------------------------------------- optimizer
def adamw(p, g, m, v, step, lr, b1, b2, eps, wd):
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    hat = m / (1 - b1 ** step)
    p = p - lr * wd * p - lr * hat / ((v / (1 - b2 ** step)).sqrt() + eps)
    return p, m, v
