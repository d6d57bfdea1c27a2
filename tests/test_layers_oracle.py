"""The 64-bit formulas that the layers' kernels are held to: their gradients against
differences of their values (on the CPU)."""
import math

import pytest
import torch

import layers_oracle as O

F64 = torch.float64


def _slopes(f, x, step=1e-6):
    """Central differences of f's scalar at x, element by element."""
    out = torch.zeros_like(x)
    flat, to = x.view(-1), out.view(-1)
    for i in range(flat.numel()):
        was = float(flat[i])
        flat[i] = was + step
        up = float(f())
        flat[i] = was - step
        to[i] = (up - float(f())) / (2 * step)
        flat[i] = was
    return out


def _near(a, b, what):
    assert torch.allclose(a, b, rtol=2e-6, atol=2e-8), (what, float((a - b).abs().max()))


def test_layer_norm():
    g = torch.Generator().manual_seed(1)
    x, dy = torch.randn(3, 7, generator=g, dtype=F64), torch.randn(3, 7, generator=g, dtype=F64)
    w, b = torch.randn(7, generator=g, dtype=F64), torch.randn(7, generator=g, dtype=F64)
    beside = torch.randn(3, 7, generator=g, dtype=F64)

    def value():
        return (O.Norm(x, w, b, 1e-3, torch.float32).y[0] * dy).sum() + (x * beside).sum()

    got = O.Norm(x, w, b, 1e-3, torch.float32).backward(dy, beside)
    for name, t in (("dx", x), ("dweight", w), ("dbias", b)):
        _near(got[name][0], _slopes(value, t), name)


@pytest.mark.parametrize("rest,mix,heat", [(False, 1.0, 1.0), (True, 1.0, 2.0), (True, 0.4, 1.5),
                                           (False, 0.0, 3.0)])
def test_distillation(rest, mix, heat):
    g = torch.Generator().manual_seed(2)
    n, classes = 5, 9
    s = torch.randn(n, classes, generator=g, dtype=F64)
    index = torch.tensor([[1, 4, 7], [0, -1, 8], [2, 2, 3], [-1, -1, -1], [9, 5, 6]], dtype=torch.int32)
    teacher = torch.randn(n, 3, generator=g, dtype=F64)
    left = torch.tensor([0.2, 0.0, 0.5, 0.3, 0.9], dtype=F64) if rest else None
    label = torch.tensor([3, -1, 2, 8, 9], dtype=torch.int32)
    dloss = torch.rand(n, generator=g, dtype=F64) + 0.5

    def of():
        return O.Distill(s, index, teacher, heat, left, label, mix, dloss, torch.float32)

    _near(of().dlogits[0], _slopes(lambda: (of().loss[0] * dloss).sum(), s), "dlogits")


def test_distillation_from_the_whole_teacher_is_a_divergence():
    """With every class named, loss = T² KL(teacher, student); its least value is 0."""
    g = torch.Generator().manual_seed(3)
    s, t = torch.randn(4, 6, generator=g, dtype=F64), torch.randn(4, 6, generator=g, dtype=F64)
    index = torch.arange(6, dtype=torch.int32).expand(4, 6).contiguous()
    one = torch.ones(4, dtype=F64)
    o = O.Distill(s, index, t, 2.0, None, None, 1.0, one, torch.float32)
    p = (t / 2).softmax(1)
    _near(o.loss[0], 4 * (p * (p.log() - (s / 2).log_softmax(1))).sum(1), "loss")
    same = O.Distill(s, index, s, 2.0, None, None, 1.0, one, torch.float32)
    assert float(same.loss[0].abs().max()) < 1e-14 and float(same.dlogits[0].abs().max()) < 1e-14


def test_distillation_of_closed_classes():
    s = torch.tensor([[0.0, -math.inf, 1.0], [-math.inf] * 3], dtype=F64)
    index = torch.tensor([[0], [1]], dtype=torch.int32)
    o = O.Distill(s, index, torch.zeros(2, 1, dtype=F64), 1.0, None, None, 1.0,
                  torch.ones(2, dtype=F64), torch.float32)
    a = math.e / (1 + math.e)
    _near(o.dlogits[0], torch.tensor([[-a, 0.0, a], [0.0, 0.0, 0.0]], dtype=F64), "dlogits")
    _near(o.loss[0], torch.tensor([-math.log(1 - a), 0.0], dtype=F64), "loss")


@pytest.mark.parametrize("gap", [0.0, 40.0, 110.0, 2000.0])
def test_distillation_whose_named_classes_lead_the_others(gap):
    """The others' share in logarithms: e^-2000 is below what 64 bits hold, its logarithm is
    not.  A difference of two losses of L, each off by up to 8 roundings of 2^-53, over 2e-6
    is off by 8 2^-53 L 10^6."""
    g = torch.Generator().manual_seed(6)
    s = torch.randn(3, 7, generator=g, dtype=F64)
    s[:, 2:] -= gap
    index = torch.tensor([[0, 1]] * 3, dtype=torch.int32)
    t, rest = torch.randn(3, 2, generator=g, dtype=F64), torch.tensor([0.3, 0.9, 0.0], dtype=F64)
    one = torch.ones(3, dtype=F64)

    def of():
        return O.Distill(s, index, t, 1.5, rest, None, 1.0, one, torch.float32)

    loga = torch.log_softmax(s / 1.5, 1)
    p = (1 - rest).unsqueeze(1) * (t / 1.5).softmax(1)
    far = torch.logsumexp(s[:, 2:] / 1.5, 1) - torch.logsumexp(s / 1.5, 1)
    share = torch.where(rest > 0, rest * (rest.clamp(min=1e-9).log() - far), 0 * rest)
    _near(of().loss[0], 2.25 * ((p * (p.log() - loga[:, :2])).sum(1) + share), "loss")
    slopes = _slopes(lambda: of().loss[0].sum(), s)
    assert torch.allclose(of().dlogits[0], slopes, rtol=2e-6,
                          atol=2e-8 + 8 * 2.0 ** -53 * float(of().loss[0].sum()) * 1e6)


@pytest.mark.parametrize("kind", ["none", "relu", "gelu", "silu"])
def test_gated_layer(kind):
    g = torch.Generator().manual_seed(4)
    x, w = torch.randn(3, 5, generator=g, dtype=F64), torch.randn(2, 4, 5, generator=g, dtype=F64)
    b, dy = torch.randn(2, 4, generator=g, dtype=F64), torch.randn(3, 4, generator=g, dtype=F64)

    def value():
        return (O.gated(x, w, b, kind, torch.float32)[0][0] * dy).sum()

    z = O.gated(x, w, b, kind, torch.float32)[1]
    got = O.gated_backward(dy, x, w, z, kind, torch.float32)
    for name, t in (("dx", x), ("dw", w), ("db", b)):
        _near(got[name][0], _slopes(value, t), name)
