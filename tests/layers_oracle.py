"""Layer norm, the gated layer, distillation and blocks of 8 bits in 64 bits, from
their definitions (no test functions here), and the bounds their kernels are held to.

Bounds as in local_oracle: V = 2^-24 is the unit roundoff of the sums, a sum of K
terms in any order is off by at most (K + 8) V times the sum of their magnitudes, a
stored value by the unit roundoff of its type.  Every function returns pairs (value,
bound).
"""
import math

import torch

import local_oracle as L
from local_oracle import V, stored


def d(t):
    return None if t is None else t.detach().double()


def close(got, want, what):
    """Every element within its bound; infinities and NaN in the same places."""
    value, bound = want
    got = got.detach().double().to(value.device)
    assert got.shape == value.shape, (what, tuple(got.shape), tuple(value.shape))
    fine = torch.isfinite(value)
    assert torch.equal(torch.isnan(got), torch.isnan(value)), (what, "NaN")
    odd = ~fine & ~torch.isnan(value)
    assert torch.equal(got[odd], value[odd]), (what, "infinities")
    over = (got - value).abs()[fine] - bound.expand_as(value)[fine]
    if over.numel() and float(over.max()) > 0:
        at = int(over.argmax())
        raise AssertionError(f"{what}: {float(got[fine][at])} for {float(value[fine][at])}, "
                             f"allowed {float(bound.expand_as(value)[fine][at]):.3e}")


# --------------------------------------------------------------- layer norm
class Norm:
    """Of x (n, width) in 64 bits; weight and bias may be None."""

    def __init__(self, x, weight, bias, eps, dtype):
        k = x.shape[1]
        self.x, self.w, self.dtype, self.k = x, weight, dtype, k
        mean = x.mean(1, keepdim=True)
        self.off = x - mean
        var = self.off.square().mean(1, keepdim=True)
        self.rstd = 1 / (var + eps).sqrt()
        # The first mean is off by `miss`; the sum of the differences from it finds that, up
        # to the differences' own roundings and their sum's.
        miss = (k + 8) * V * x.abs().mean(1, keepdim=True)
        around = self.off.abs().mean(1, keepdim=True) + miss
        self.centre = (k + 8) * V * around + 4 * V * miss
        var_err = (k + 12) * V * (var + miss.square()) + 2 * self.centre * around
        # rstd: half the relative error of var + eps, and its own places
        self.rho = (var_err / (var + eps)).clamp(max=1.0) + 4 * V
        self.mean = (mean, self.centre + V * mean.abs() + 4 * V * miss)
        self.xh = self.off * self.rstd
        slack = self.rstd * (self.centre + 4 * V * self.off.abs()) + self.xh.abs() * self.rho
        scale = 1.0 if weight is None else weight.abs()
        y = self.xh if weight is None else self.xh * weight
        err = slack * scale + 4 * V * y.abs()
        if bias is not None:
            y = y + bias
            err = err + 2 * V * bias.abs()
        self.y = (y, err + stored(y, dtype))
        # backward reads the mean as rounded
        self.xh_err = self.rstd * (self.mean[1] + 4 * V * self.off.abs()) + self.xh.abs() * self.rho

    def backward(self, dy, beside, found=False):
        """{"dx", "dweight", "dbias"}.  found: the mean's rounding is found from the row's
        differences from it and taken out."""
        n, k = dy.shape
        xh, e, shift = self.xh, self.xh_err, 0.0
        if found:
            # the rounded mean is off by `miss`; the differences' sum finds that but for its
            # roundings and theirs, and xh of the rounded mean is `shift` larger
            miss = V * self.mean[0].abs() + self.mean[1]
            centre = (k + 8) * V * (self.off.abs().mean(1, keepdim=True) + miss)
            e = self.rstd * (centre + 6 * V * (self.off.abs() + miss)) + xh.abs() * self.rho
            shift = self.rstd * miss
        g = dy if self.w is None else dy * self.w
        s0, e0 = g.mean(1, keepdim=True), (k + 8) * V * g.abs().mean(1, keepdim=True)
        s1 = (g * xh).mean(1, keepdim=True)
        e1 = ((k + 8) * V * g.abs() * (xh.abs() + shift) + g.abs() * e).mean(1, keepdim=True)
        e1 = e1 + shift * (e0 + 4 * V * s0.abs())
        dx = self.rstd * (g - s0 - xh * s1)
        size = self.rstd * (g.abs() + s0.abs() + (xh.abs() + shift) * s1.abs())
        err = self.rstd * (e0 + (xh.abs() + shift) * e1 + e * (s1.abs() + e1)) + (self.rho + 8 * V) * size
        if beside is not None:
            dx = dx + beside
            err = err + 2 * V * beside.abs()
        dw, db = (dy * xh).sum(0), dy.sum(0)
        dw_err = (n + 8) * V * (dy * xh).abs().sum(0) + (dy.abs() * e).sum(0)
        db_err = (n + 8) * V * dy.abs().sum(0)
        return {"dx": (dx, err + stored(dx, self.dtype)),
                "dweight": (dw, dw_err + stored(dw, self.dtype)),
                "dbias": (db, db_err + stored(db, self.dtype))}


# ------------------------------------------------------------- distillation
class Distill:
    """loss (n,) and dlogits (n, classes) with their bounds.  index (n, k) with entries
    outside [0, classes) absent, teacher (n, k) in 64 bits, rest, label may be None."""

    def __init__(self, s, index, teacher, heat, rest, label, mix, dloss, dtype):
        n, classes = s.shape
        zero = torch.zeros(n, 1, dtype=torch.float64, device=s.device)
        shut = ~(s > -math.inf).any(1, keepdim=True) & ~torch.isnan(s).any(1, keepdim=True)
        top = s.max(1, keepdim=True).values
        u = torch.where(shut, zero, (s - top) / heat)
        e, self.loss_err = u.exp(), 0

        def weighed(e, u):      # a sum of exponentials, and its relative error
            z = e.sum(1, keepdim=True)
            slack = (e * (u.abs().nan_to_num(posinf=0.0) * 4 + 8)).sum(1, keepdim=True) * V
            return z, slack / torch.where(z > 0, z, z + 1) + (classes + 8) * V

        z, dz = weighed(e, u)
        a = e / z
        da = (u.abs().nan_to_num(posinf=0.0) * 4 + 10) * V + dz
        soft, soft_err = zero, zero
        grad = torch.zeros_like(s)
        grad_err = torch.zeros_like(s)
        scale = dloss.unsqueeze(1)
        if index is not None and mix != 0:
            k = index.shape[1]
            there = (index >= 0) & (index < classes)
            at = index.long().clamp(0, classes - 1)
            t = torch.where(there, teacher / heat, torch.full_like(teacher, -math.inf))
            odd = torch.isnan(t).any(1, keepdim=True) | (t == math.inf).any(1, keepdim=True)
            taught = (t > -math.inf).any(1, keepdim=True) | odd
            best = torch.where(taught, t.max(1, keepdim=True).values, zero)
            q = (t - best).exp()
            total = q.sum(1, keepdim=True)
            r = zero if rest is None else torch.where(taught, rest.unsqueeze(1).clamp(min=0, max=1), zero)
            p = (1 - r) * q / torch.where(taught, total, total + 1)
            dp = ((t - best).abs().nan_to_num(posinf=0.0) * 4 + k + 14) * V
            dp = dp.max(1, keepdim=True).values + dp
            live = there & (p != 0) | odd
            ut = u.gather(1, at)
            loga = ut - z.log()
            dlog = (ut.abs().nan_to_num(posinf=0.0) * 6 + 4 * z.log().abs()) * V + dz
            term = torch.where(live, p * (torch.where(live, p, p * 0 + 1).log() - loga), p * 0)
            away = (p.clamp(min=1e-300).log().abs() + loga.abs().nan_to_num(posinf=0.0))
            wobble = torch.where(live, p * (dp * (away + 1) + dlog + 4 * V * away), p * 0)
            soft = term.sum(1, keepdim=True)
            soft_err = wobble.sum(1, keepdim=True) + (k + 8) * V * term.abs().sum(1, keepdim=True)
            member = torch.zeros(n, classes + 1, dtype=torch.bool, device=s.device)
            member.scatter_(1, torch.where(there, at, classes), True)
            member = member[:, :classes]
            # the classes left out, from the largest of them: their share of z can be far
            # below what 64 bits hold
            ur = torch.where(member, zero - math.inf, u)
            lead = ur.max(1, keepdim=True).values
            open_ = lead > -math.inf
            lead = torch.where(open_ | torch.isnan(lead), lead, zero)
            er = (ur - lead).exp()
            # the exponents count from the row's maximum or from theirs: from the row's, where
            # they leave no more than 2^-60 of its sum, they lose too many
            off = (ur - lead).abs() + lead.abs().clamp(max=60 * math.log(2))
            zr, dzr = weighed(er, off)
            log_ar = lead + zr.log() - z.log()
            has = r > 0
            safe = torch.where(has, r, zero + 1)
            left = safe * (safe.log() - log_ar)
            soft = soft + torch.where(has, left, zero)
            soft_err = soft_err + torch.where(
                has, safe * (dz + dzr + 8 * V * (safe.log().abs() + lead.abs() + zr.log().abs()
                                                 + z.log().abs())),
                zero).nan_to_num(posinf=0.0)
            soft = torch.where(taught, soft, zero)
            soft = torch.where(odd, zero * math.nan, soft)
            given = torch.zeros(n, classes + 1, dtype=torch.float64, device=s.device)
            given.scatter_add_(1, torch.where(there, at, classes), torch.where(there, p, p * 0))
            given = given[:, :classes]
            of_rest = torch.where(has & open_, r * er / torch.where(open_, zr, zr + 1), zero)
            g = torch.where(member, a - given, torch.where(torch.isinf(ur), a, a - of_rest))
            ge = torch.where(member, a * da + given * (dp.max(1, keepdim=True).values + k * V),
                             a * da + of_rest * (dz + dzr + (off.nan_to_num(posinf=0.0) * 4 + 16) * V))
            ge = ge + 6 * V * (a + of_rest + given)
            # The hardware's exponential has no subnormals: what is below 2^-126 is 0.  a, of a
            # sum of 1 or more, is off by as much; a share of the rest, of a sum of 2^-60 or
            # more (or from its own maximum), by up to 2^-126 / 2^-60 of it.
            ge = ge + 2.0 ** -126 + torch.where(has & open_ & ~member, r * 2.0 ** -66, zero)
            g = torch.where(odd, g * math.nan, g)
            grad = torch.where(taught, mix * heat * g, zero)
            grad_err = torch.where(taught, mix * heat * ge, zero)
        loss = mix * heat * heat * soft if mix != 0 else zero
        loss_err = mix * heat * heat * (soft_err + 4 * V * soft.abs())
        if label is not None and mix != 1:
            known = ((label >= 0) & (label < classes)).unsqueeze(1)
            which = label.long().clamp(0, classes - 1).unsqueeze(1)
            u1 = torch.where(shut, zero, s - top)
            e1 = u1.exp()
            z1, dz1 = weighed(e1, u1)
            a1 = e1 / z1
            ul = u1.gather(1, which)
            hard = z1.log() - ul
            hard_err = dz1 + 6 * V * (z1.log().abs() + ul.abs().nan_to_num(posinf=0.0))
            loss = loss + torch.where(known, (1 - mix) * hard, zero)
            loss_err = loss_err + torch.where(known, (1 - mix) * hard_err, zero)
            one = torch.zeros_like(s).scatter_(1, which, 1.0)
            da1 = (u1.abs().nan_to_num(posinf=0.0) * 4 + 10) * V + dz1
            grad = grad + torch.where(known, (1 - mix) * (a1 - one), zero)
            grad_err = grad_err + torch.where(
                known, (1 - mix) * (a1 * da1 + 6 * V * (a1 + one) + 2.0 ** -126), zero)
        loss = torch.where(shut, zero, loss).squeeze(1)
        grad = torch.where(shut, zero, grad) * scale
        grad_err = torch.where(shut, zero, grad_err) * scale.abs() + 8 * V * grad.abs()
        # the loss is fp32: beyond its largest number, (2 - 2^-24) 2^127 with half a step, it
        # rounds to infinity
        loss = torch.where(loss >= (2 - 2.0 ** -24) * 2.0 ** 127, loss * math.inf, loss)
        tiny = 2.0 ** -140      # sums and products next to fp32's least value
        self.loss = (loss, (loss_err.squeeze(1) + 8 * V * loss.abs() + tiny).nan_to_num(posinf=0.0))
        self.dlogits = (grad, (grad_err + stored(grad, dtype) + tiny).nan_to_num(posinf=0.0))


# -------------------------------------------------------------- gated layer
def gated(x, w, b, kind, dtype):
    """((y, bound), (z, bound)) with z (n, 2, hidden)."""
    k, hidden = x.shape[1], w.shape[1]
    flat = w.reshape(2 * hidden, k)
    z = x @ flat.t()
    size = x.abs() @ flat.abs().t()
    if b is not None:
        z, size = z + b.reshape(-1), size + b.abs().reshape(-1)
    zerr = (k + 8) * V * size
    u, v = z[:, :hidden], z[:, hidden:]
    h, herr = L.act(u, kind), L.SLOPE[kind] * zerr[:, :hidden] + 8 * V * u.abs()
    y = h * v
    err = herr * (v.abs() + zerr[:, hidden:]) + h.abs() * zerr[:, hidden:] + 4 * V * y.abs()
    n = x.shape[0]
    return (y, err + stored(y, dtype)), (z.view(n, 2, hidden), zerr.view(n, 2, hidden))


def held(dz):
    """How far fp16 is off that holds dz over a power of two with which the largest
    magnitude lies in [2^14, 2^15), unless it lies in [1/4, 65,520) already: half a step,
    2^-11 of the value or 2^-25 and the power, whichever is more."""
    size = dz.abs()
    largest = float(torch.where(torch.isfinite(size), size, size * 0).max()) if size.numel() else 0.0
    power = 0
    if largest and not 0.2499 <= largest < 65600:      # next to the ends either is right
        power = math.frexp(largest)[1] - 14
    return torch.maximum(size * 2.0 ** -11, torch.full_like(size, 2.0 ** (power - 25)))


def gated_backward(dy, x, w, z, kind, dtype, powers=False):
    """{"dx", "dw", "db"} from z = (value, bound).  powers: fp16's dz is held over a power of
    two (held), not as it is."""
    n, k = x.shape
    hidden = w.shape[1]
    u, v = z[0][:, 0], z[0][:, 1]
    ue, ve = z[1][:, 0], z[1][:, 1]
    slope, h = L.act_slope(u, kind), L.act(u, kind)
    se = L.BEND[kind] * ue + 16 * V
    if kind == "relu":      # next to the kink either slope is right
        se = se + (u.abs() <= ue).double()
    he = L.SLOPE[kind] * ue + 8 * V * u.abs()
    dz = torch.cat([dy * v * slope, dy * h], 1)
    raw = torch.cat([dy.abs() * (se * (v.abs() + ve) + slope.abs() * ve), dy.abs() * he], 1)
    raw = raw + 4 * V * dz.abs()
    err = raw + (held(dz) if powers else stored(dz, dtype))      # for the two products
    flat = w.reshape(2 * hidden, k)
    dx, dw, db = dz @ flat, dz.t() @ x, dz.sum(0)
    dx_err = (2 * hidden + 8) * V * (dz.abs() @ flat.abs()) + err @ flat.abs()
    dw_err = (n + 8) * V * (dz.abs().t() @ x.abs()) + err.t() @ x.abs()
    db_err = (n + 8) * V * dz.abs().sum(0) + raw.sum(0)
    return {"dx": (dx, dx_err + stored(dx, dtype)),
            "dw": ((dw).view(2, hidden, k), (dw_err + stored(dw, dtype)).view(2, hidden, k)),
            "db": (db.view(2, hidden), (db_err + stored(db, dtype)).view(2, hidden))}


# ------------------------------------------------------------ blocks of 8 bits
BLOCK = 128


def blocks(x):
    """(values, exponents): what e4m3 holds of the rows of x (n, width) with a power of
    two to 128 neighbours, each rounded to the nearest, ties to even.  In 64 bits every
    step is exact."""
    n, width = x.shape
    count = -(-width // BLOCK)
    full = torch.zeros(n, count * BLOCK, dtype=torch.float64, device=x.device)
    full[:, :width] = x
    full = full.view(n, count, BLOCK)
    size = torch.where(torch.isfinite(full), full.abs(), torch.zeros_like(full)).amax(2)
    m, e = torch.frexp(size)                    # size = m 2^e, 1/2 <= m < 1; 448 = 0.875 2^9
    e = torch.where(size > 0, e - 9 + (m > 0.875).int(), torch.full_like(e, -126)).clamp(min=-126)
    u = full * torch.exp2(-e.double()).unsqueeze(2)
    finite = torch.isfinite(u)
    step = torch.exp2(torch.floor(torch.log2(torch.where(finite, u.abs(), u * 0 + 1).clamp(min=2.0 ** -6))) - 3)
    held = torch.where(finite, (u / step).round() * step, torch.full_like(u, math.nan))
    return (held * torch.exp2(e.double()).unsqueeze(2)).view(n, -1)[:, :width], e


def linear8(x, w, b, kind, r, dtype):
    """(y, bound) of a product of held values x (n, inner) and w (outer, inner).

    The matrix instruction brings eight neighbouring products at a time to the largest
    one's exponent and drops what lies 13 bits below it: each of the eight is off by less
    than 2^-13 of the power of two at or below the largest, all by at most 2^-10 of it."""
    n, inner = x.shape
    pad = -inner % 8
    xs = torch.nn.functional.pad(x, (0, pad)).view(n, 1, -1, 8)
    ws = torch.nn.functional.pad(w, (0, pad)).view(1, w.shape[0], -1, 8)
    most = torch.zeros(n, w.shape[0], dtype=torch.float64, device=x.device)
    for i in range(0, n, 64):       # eight products at a time, of 64 rows
        most[i:i + 64] = (xs[i:i + 64] * ws).abs().amax(3).sum(2)
    z = x @ w.t() + (0 if b is None else b)
    size = x.abs() @ w.abs().t() + (0 if b is None else b.abs())
    zerr = 2.0 ** -10 * most + (inner + 8) * V * size
    y = L.act(z, kind)
    err = L.SLOPE[kind] * zerr + 8 * V * z.abs()
    if r is not None:
        y = y + r
        err = err + 4 * V * r.abs()
    return y, err + stored(y, dtype)
