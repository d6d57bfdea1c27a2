"""Layer norm, the gated layer, distillation and blocks of 8 bits in 64 bits, from
their definitions (no test functions here), and the bounds their kernels are held to.

Bounds as in local_oracle: V = 2^-24 is the unit roundoff of the sums, a sum of K
terms in any order is off by at most (K + 8) V times the sum of their magnitudes, a
stored value by the unit roundoff of its type.  Every function returns pairs (value,
bound).
"""
import math

import torch

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

    def backward(self, dy, beside):
        """{"dx", "dweight", "dbias"}"""
        n, k = dy.shape
        xh, e = self.xh, self.xh_err
        g = dy if self.w is None else dy * self.w
        s0, e0 = g.mean(1, keepdim=True), (k + 8) * V * g.abs().mean(1, keepdim=True)
        s1 = (g * xh).mean(1, keepdim=True)
        e1 = ((k + 8) * V * (g * xh).abs() + g.abs() * e).mean(1, keepdim=True)
        dx = self.rstd * (g - s0 - xh * s1)
        size = self.rstd * (g.abs() + s0.abs() + (xh * s1).abs())
        err = self.rstd * (e0 + xh.abs() * e1 + e * (s1.abs() + e1)) + (self.rho + 8 * V) * size
        if beside is not None:
            dx = dx + beside
            err = err + 2 * V * beside.abs()
        dw, db = (dy * xh).sum(0), dy.sum(0)
        dw_err = (n + 8) * V * (dy * xh).abs().sum(0) + (dy.abs() * e).sum(0)
        db_err = (n + 8) * V * dy.abs().sum(0)
        return {"dx": (dx, err + stored(dx, self.dtype)),
                "dweight": (dw, dw_err + stored(dw, self.dtype)),
                "dbias": (db, db_err + stored(db, self.dtype))}
