"""Layer norm, gated layer, residual, head and distillation from a map as one model:
its gradients against 64 bits and against differences, its training step in a graph,
and its head in 8 bits."""
import pytest
import torch

import layers_oracle as O
from gpu_util import torch_cuda
from paper_1905_09598_amd import local

pytestmark = pytest.mark.gpu
F64 = torch.float64


class Student:
    """scores = head(h w2 + b2 + x), h the gated layer of the normed x."""

    def __init__(self, d, hidden, classes, dtype, seed=0):
        g = torch.Generator().manual_seed(seed)

        def draw(*shape, scale):
            return (scale * torch.randn(*shape, generator=g)).to(dtype).cuda()

        self.params = [(1 + draw(d, scale=0.1).float()).to(dtype), draw(d, scale=0.1),
                       draw(2, hidden, d, scale=d ** -0.5), draw(2, hidden, scale=0.1),
                       draw(d, hidden, scale=hidden ** -0.5), draw(d, scale=0.1),
                       draw(classes, d, scale=d ** -0.5), draw(classes, scale=0.1)]

    def step(self, x, said, dloss):
        """(loss, scores, gradients of the parameters, of x)"""
        nw, nb, w1, b1, w2, b2, wh, bh = self.params
        y, kept = local.norm(x, nw, nb, keep=True)
        h, z = local.gated(y, w1, b1, keep=True)
        u = local.linear(h, w2, b2, residual=x)
        s = local.linear(u, wh, bh)
        loss, ds = local.distill(s, *said, dloss=dloss)
        du, dwh, dbh = local.linear_backward(ds, u, wh)
        dh, dw2, db2 = local.linear_backward(du, h, w2)
        dy, dw1, db1 = local.gated_backward(dh, y, w1, z)
        dx, dnw, dnb = local.norm_backward(dy, x, nw, kept, du)
        return loss, s, [dnw, dnb, dw1, db1, dw2, db2, dwh, dbh], dx

    def loss(self, x, said):
        nw, nb, w1, b1, w2, b2, wh, bh = self.params
        u = local.linear(local.gated(local.norm(x, nw, nb), w1, b1), w2, b2, residual=x)
        return local.distill(local.linear(u, wh, bh), *said)


def _said(n, classes, seed=1):
    """What a map of `classes` units says: its four best, their scores, the rest, and
    labels beside it, at temperature 2."""
    g = torch.Generator().manual_seed(seed)
    scores = (2 * torch.randn(n, classes, generator=g)).cuda()
    r = local.route(scores / 2, 4, renormalise=False)
    t = scores.gather(1, r.index.long())
    label = torch.randint(-1, classes, (n,), generator=g).int().cuda()
    return r.index, t, 2.0, (1 - r.weight.sum(1)).clamp(min=0), label, 0.7


def _exact(student, x, said, dloss):
    p = [v.double().requires_grad_() for v in student.params]
    x = x.double().requires_grad_()
    nw, nb, w1, b1, w2, b2, wh, bh = p
    off = x - x.mean(1, keepdim=True)
    y = off * torch.rsqrt(off.square().mean(1, keepdim=True) + 1e-5) * nw + nb
    u, v = y @ w1[0].t() + b1[0], y @ w1[1].t() + b1[1]
    s = (u * torch.sigmoid(u) * v @ w2.t() + b2 + x) @ wh.t() + bh
    index, t, heat, rest, label, mix = said
    o = O.Distill(s.detach(), index, O.d(t), heat, O.d(rest), label, mix, O.d(dloss), torch.float32)
    grads = torch.autograd.grad(s, p + [x], o.dlogits[0])
    return o.loss[0], s.detach(), grads[:-1], grads[-1]


def _off(a, b):
    return float((a.double() - b).norm() / b.norm())


# The largest relative error (2-norm).  fp32: sums of up to 520 terms, a dozen in a chain.
# 16 bits: about a dozen roundings of half a step (0.29 of it in the mean: bf16 2^-8 0.58)
# between x and a gradient, and the softmax's slope doubles what the scores are off by.
@pytest.mark.parametrize("dtype,bound", [(torch.float32, 2e-5), (torch.bfloat16, 0.03),
                                         (torch.float16, 0.004)])
@pytest.mark.parametrize("n,d,hidden,classes", [(1, 64, 40, 30), (70, 200, 129, 100),
                                                (600, 520, 264, 400)])
def test_gradients(n, d, hidden, classes, dtype, bound):
    torch_cuda()
    student, said = Student(d, hidden, classes, dtype), _said(n, classes)
    g = torch.Generator().manual_seed(5)
    x, dloss = torch.randn(n, d, generator=g).to(dtype).cuda(), (0.5 + torch.rand(n, generator=g)).cuda()
    got, want = student.step(x, said, dloss), _exact(student, x, said, dloss)
    assert _off(got[1], want[1]) < bound and _off(got[0], want[0]) < bound
    for i, (u, v) in enumerate(zip(got[2], want[2])):
        assert _off(u, v) < bound, (i, _off(u, v))
    assert _off(got[3], want[3]) < bound
    assert torch.equal(student.loss(x, said), got[0])


def test_gradients_against_differences():
    """In fp32 along one direction of all parameters: the third derivative's part of a
    central difference of step 2^-7 is below 2^-14 of curvatures of about one, the losses'
    roundings, 2^-24 of 64 losses of about 3 over 2^-6, below 2^-11."""
    student, said = Student(96, 64, 50, torch.float32), _said(64, 50)
    x = torch.randn(64, 96, generator=torch.Generator().manual_seed(6)).cuda()
    _, _, grads, _ = student.step(x, said, torch.ones(64, device="cuda"))
    g = torch.Generator().manual_seed(7)
    way = [torch.randn(p.shape, generator=g).cuda() for p in student.params]
    size = sum(float(v.double().square().sum()) for v in way) ** 0.5
    way = [v / size for v in way]
    slope = sum(float((a.double() * v.double()).sum()) for a, v in zip(grads, way))
    step, ends, at = 2.0 ** -7, [], [p.clone() for p in student.params]
    for sign in (1, -1):
        for p, b, v in zip(student.params, at, way):
            p.copy_(b + sign * step * v)
        ends.append(float(student.loss(x, said).double().sum()))
    assert abs((ends[0] - ends[1]) / (2 * step) - slope) < 2.0 ** -9 * max(1.0, abs(slope))


def test_a_training_step_in_a_graph():
    """Captured and replayed with the program's own calls between, against eager steps."""
    def made():
        s = Student(128, 96, 60, torch.bfloat16)
        return s, local.AdamW(s.params, lr=1e-2, bits=8, master=True)

    (a, opt_a), (b, opt_b) = made(), made()
    said, dloss = _said(200, 60), torch.full((200,), 1 / 200, device="cuda")
    x = torch.randn(200, 128, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    graph = torch.cuda.CUDAGraph()
    b.step(x, said, dloss)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = b.step(x, said, dloss)
    for k in range(4):
        x.copy_(torch.randn(200, 128, generator=torch.Generator().manual_seed(k)).bfloat16())
        eager = a.step(x, said, dloss)
        graph.replay()
        for u, v in zip([eager[0], eager[1], *eager[2], eager[3]],
                        [held[0], held[1], *held[2], held[3]]):
            assert torch.equal(u, v), k
        opt_a.step(eager[2])
        opt_b.step(held[2])
        torch.cuda.synchronize()
    for u, v in zip(a.params, b.params):
        assert torch.equal(u, v)
    assert not torch.equal(a.params[2], Student(128, 96, 60, torch.bfloat16).params[2])


@pytest.mark.parametrize("n", [1, 300])
def test_the_head_in_8_bits(n):
    """Two operands rounded to e4m3, off by up to 2^-4 and 0.58 of it in the mean each: the
    scores by less than 2^-4 in all."""
    student = Student(520, 264, 400, torch.bfloat16)
    nw, nb, w1, b1, w2, b2, wh, bh = student.params
    x = torch.randn(n, 520, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    u = local.linear(local.gated(local.norm(x, nw, nb), w1, b1), w2, b2, residual=x)
    s, s8 = local.linear(u, wh, bh), local.linear8(u, local.to_blocks(wh), bh)
    assert 0 < _off(s8, s.double()) < 2.0 ** -4
    index = local.route(s8, 4).index
    assert index.shape == (n, 4) and int(index.min()) >= 0
