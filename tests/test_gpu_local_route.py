"""Routing, dispatch and their gradients against the definitions in 64 bits."""
import math

import pytest
import torch

import local_oracle as O
from gpu_util import say, torch_cuda
from paper_1905_09598_amd import local

pytestmark = pytest.mark.gpu
T = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
INF = math.inf


def _scores(n, experts, dtype, seed=0, closed=0.0):
    g = torch.Generator().manual_seed(seed)
    s = torch.randn(n, experts, generator=g) * 2
    if closed:
        s[torch.rand(n, experts, generator=g) < closed] = -INF
    return s.to(dtype).cuda()


def _order(index, experts):
    """offsets, order and place of an assignment, slot by slot."""
    flat = index.flatten().tolist()
    rows = [[s for s, e in enumerate(flat) if e == x] for x in range(experts)]
    offsets, order = [0], []
    for r in rows:
        order += r
        offsets.append(len(order))
    place = [-1] * len(flat)
    for p, s in enumerate(order):
        place[s] = p
    return offsets, order + [-1] * (len(flat) - len(order)), place


def _check(scores, k, bias=None, order=True, **how):
    r = local.route(scores, k, bias, **how)
    index, weight = O.route(scores.cpu(), k, None if bias is None else bias.cpu(), **how)
    assert torch.equal(r.index.cpu().long(), index)
    # each factor within a few fp32 roundings: e^x of an argument that is off by 2 v |x|,
    # and sums of up to `experts` terms
    n, experts = scores.shape
    span = scores.float()
    span = float(span[span.isfinite()].abs().max()) if span.isfinite().any() else 0.0
    bound = (16 + 4 * span + (experts if how.get("gate") != "sigmoid" else 64)) * O.V
    O.close(r.weight, (weight, bound * weight.abs() + 2.0 ** -126), "weight")
    if order:
        want = _order(r.index.cpu(), experts)
        for got, w in zip((r.offsets, r.order, r.place), want):
            assert got.cpu().tolist() == w
    return r, index


# below, at and beyond 16 lanes and a wave; each instance of the kernel
SIZES = [(1, 1, 1), (1, 64, 2), (3, 5, 5), (33, 64, 6), (20, 100, 4), (17, 256, 8), (9, 257, 16),
         (9, 400, 3), (5, 513, 17), (4, 2048, 64), (3, 2049, 5), (2, 10000, 8)]


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("gate", list(local.GATES))
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("n,experts,k", SIZES)
def test_choice_and_weights(n, experts, k, renormalise, gate, dtype):
    torch_cuda()
    say("route", n, experts, k, renormalise, gate, dtype)
    _check(_scores(n, experts, T[dtype], seed=experts, closed=0.2), k, gate=gate,
           renormalise=renormalise, scale=1.7)


@pytest.mark.parametrize("gate", list(local.GATES))
@pytest.mark.parametrize("group_best", [1, 2])
@pytest.mark.parametrize("experts,groups,top,k", [(8, 8, 3, 3), (64, 4, 2, 8), (240, 8, 3, 5),
                                                  (256, 16, 4, 8), (320, 64, 10, 20),
                                                  (2100, 7, 2, 6), (96, 3, 3, 4)])
def test_groups_and_bias(experts, groups, top, k, group_best, gate):
    g = torch.Generator().manual_seed(experts)
    bias = (0.3 * torch.randn(experts, generator=g)).cuda()
    bias[1] = -INF                                    # an expert taken out of service
    _check(_scores(25, experts, torch.float32, seed=groups, closed=0.3), k, bias, gate=gate,
           groups=groups, top_groups=top, group_best=group_best)


@pytest.mark.parametrize("experts", [64, 400, 3000])
@pytest.mark.parametrize("gate", list(local.GATES))
def test_equal_scores_go_to_the_lowest_expert(experts, gate):
    s = torch.zeros(6, experts, device="cuda")
    s[1, 5::7] = 1
    s[2] = torch.finfo(torch.float32).min     # the type's lowest value is a score like any other
    s[3, :] = -0.0
    s[3, 1::2] = 0.0
    s[4, 3] = torch.finfo(torch.float32).min
    r, index = _check(s, 4, gate=gate)
    assert index[0].tolist() == [0, 1, 2, 3] and index[1].tolist() == [5, 12, 19, 26]
    assert index[2].tolist() == [0, 1, 2, 3]


@pytest.mark.parametrize("experts", [12, 300, 2500])
@pytest.mark.parametrize("gate", list(local.GATES))
@pytest.mark.parametrize("renormalise", [True, False])
def test_rows_without_an_open_expert_and_spoilt_rows(experts, gate, renormalise):
    s = _scores(9, experts, torch.float32, seed=1)
    s[0] = -INF
    s[2, 1:] = -INF                     # one expert left
    s[3, 4] = float("nan")
    s[5, 6] = INF
    s[6] = -INF
    s[6, 2] = float("nan")
    r, index = _check(s, 3, gate=gate, renormalise=renormalise)
    assert index[0].tolist() == [-1] * 3 and index[2].tolist() == [0, -1, -1]
    dw = torch.ones(9, 3, device="cuda")
    ds = local.route_backward(dw, s, r).cpu()
    assert not ds[0].any() and torch.isnan(ds[3]).all() and torch.isnan(ds[6]).all()
    assert torch.isfinite(ds[[1, 2, 4, 7, 8]]).all()
    assert torch.isnan(ds[5]).all() == (gate == "softmax")


@pytest.mark.parametrize("n,experts,k", [(0, 8, 2), (1, 1, 1)])
def test_no_rows_and_one_expert(n, experts, k):
    s = _scores(n, experts, torch.bfloat16)
    r = local.route(s, k)
    assert r.index.shape == (n, k) and r.offsets.cpu()[-1] == n * k
    assert torch.equal(r.weight.cpu(), torch.ones(n, k))
    assert local.route_backward(r.weight, s, r).shape == (n, experts)


def test_strided_scores():
    wide = torch.full((40, 131), float("nan"), device="cuda")
    s = wide[:, 3:103]
    s.copy_(_scores(40, 100, torch.float32, seed=8))
    a, b = local.route(s, 5), local.route(s.contiguous(), 5)
    assert torch.equal(a.index, b.index) and torch.equal(a.weight, b.weight)
    d = torch.randn(40, 5, device="cuda")
    assert torch.equal(local.route_backward(d, s, a), local.route_backward(d, s.contiguous(), b))


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("gate", list(local.GATES))
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("n,experts,k", [(1, 3, 2), (40, 64, 4), (21, 512, 16), (9, 700, 20),
                                         (3, 2500, 8)])
def test_gradient(n, experts, k, renormalise, gate, dtype):
    scale = 1.3
    s = _scores(n, experts, T[dtype], seed=n, closed=0.1)
    r = local.route(s, k, gate=gate, renormalise=renormalise, scale=scale)
    g = torch.Generator().manual_seed(3)
    for gt in (torch.float32, T[dtype]):
        dw = torch.randn(n, k, generator=g).to(gt).cuda()
        got = local.route_backward(dw, s, r)
        s64 = O.d(s).requires_grad_()
        index = r.index.cpu().long()
        w = O.route_weight(s64, index, gate, renormalise, scale)
        (w * O.d(dw)).sum().backward()
        # a difference of terms up to |g| w each, in fp32
        mag = scale * (O.d(dw).abs() * (index >= 0)).sum(1, keepdim=True)
        O.close(got, (s64.grad.nan_to_num(0.0),
                      64 * O.V * mag + O.stored(s64.grad.nan_to_num(0.0), T[dtype])), "dscores")


@pytest.mark.parametrize("gate", list(local.GATES))
def test_one_renormalised_choice_has_no_gradient(gate):
    s = _scores(200, 9, torch.float32, seed=4)
    r = local.route(s, 1, gate=gate, scale=1.7)
    assert not local.route_backward(torch.randn(200, 1, device="cuda"), s, r).any()


def test_gradient_is_the_slope_of_the_loss():
    for gate in local.GATES:
        for renormalise in (True, False):
            s = _scores(12, 30, torch.float32, seed=6)
            r = local.route(s, 4, gate=gate, renormalise=renormalise, scale=2.0)
            g = torch.Generator().manual_seed(1)
            dw, v = torch.randn(12, 4, generator=g), torch.randn(12, 30, generator=g).double()
            ds = O.d(local.route_backward(dw.cuda(), s, r))
            index = r.index.cpu().long()

            def loss(t):
                w = O.route_weight(O.d(s) + t * v, index, gate, renormalise, 2.0)
                return float((w * dw.double()).sum())

            slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
            assert abs(float((ds * v).sum()) - slope) <= 1e-5 * (1 + abs(slope))


@pytest.mark.parametrize("n,k,experts", [(1, 1, 1), (7, 3, 5), (64, 1, 2), (2000, 2, 100),
                                         (4096, 1, 7), (5000, 3, 2000), (9000, 2, 300),
                                         (6000, 2, 5000), (3, 2, 16384)])
def test_dispatch(n, k, experts):
    g = torch.Generator().manual_seed(n)
    index = torch.randint(-1, experts, (n, k), generator=g, dtype=torch.int32)
    if n > 100:                       # popular experts, and one without documents
        index[torch.rand(n, k, generator=g) < 0.5] = experts // 2
        index[index == experts // 3] = -1
    r = local.dispatch(index.cuda(), None, experts)
    flat = index.flatten().long()
    key = torch.where(flat < 0, torch.full_like(flat, experts), flat)
    order = torch.sort(key, stable=True).indices
    there = int((flat >= 0).sum())
    count = torch.bincount(key, minlength=experts + 1)[:experts]
    assert torch.equal(r.offsets.cpu().long(), torch.cat([torch.zeros(1).long(), count.cumsum(0)]))
    assert torch.equal(r.order.cpu().long()[:there], order[:there])
    assert (r.order.cpu()[there:] == -1).all()
    place = torch.full_like(flat, -1)
    place[order[:there]] = torch.arange(there)
    assert torch.equal(r.place.cpu().long(), place)
    assert torch.equal(r.load.cpu().long(), count)


@pytest.mark.parametrize("n,experts,k", [(1, 64, 2), (16, 256, 4), (17, 256, 4), (4, 300, 16),
                                         (5, 300, 3), (1, 2048, 64), (2, 100, 40), (3, 20, 20),
                                         (16, 30, 5)])
def test_few_slots_are_sorted_with_the_routing(n, experts, k):
    s = _scores(n, experts, torch.bfloat16, seed=n + k, closed=0.5)
    s[n // 2] = -INF
    if n > 2:
        s[0, 0] = float("nan")
    r, _ = _check(s, k)
    again = local.dispatch(r.index, r.weight, experts)
    for name in ("offsets", "order", "place"):
        assert torch.equal(getattr(r, name), getattr(again, name))


def test_dispatch_counts_strange_entries_as_absent():
    index = torch.tensor([[0, 7], [-5, 2], [3, 1 << 30]], dtype=torch.int32).cuda()
    r = local.dispatch(index, None, 3)
    assert r.offsets.cpu().tolist() == [0, 1, 1, 2]
    assert r.order.cpu().tolist() == [0, 3, -1, -1, -1, -1]
    assert r.place.cpu().tolist() == [0, -1, -1, 1, -1, -1]


@pytest.mark.parametrize("n,k,experts", [(300_000, 1, 9), (20_000, 2, 4000), (9000, 40, 300)])
def test_dispatch_of_many_slots(n, k, experts):
    # the order of a stable sort; absent slots behind all others
    g = torch.Generator().manual_seed(n)
    index = torch.randint(-1, experts, (n, k), generator=g, dtype=torch.int32)
    r = local.dispatch(index.cuda(), None, experts)
    key = index.flatten().long()
    count = torch.bincount(key[key >= 0], minlength=experts)
    assert torch.equal(r.offsets.cpu().long()[1:], count.cumsum(0)) and r.offsets[0] == 0
    order = torch.sort(torch.where(key < 0, experts, key), stable=True).indices
    there = int(count.sum())
    assert torch.equal(r.order.cpu().long()[:there], order[:there])
    assert (r.order[there:] == -1).all()
    place = torch.full((n * k,), -1)
    place[order[:there]] = torch.arange(there)
    assert torch.equal(r.place.cpu().long().flatten(), place)


def test_rows_beyond_one_launch():
    # a block of rows over and over: its answers over and over
    g = torch.Generator().manual_seed(8)
    block = torch.randn(1000, 4, generator=g).cuda()
    n = 8_400_000
    scores = block.repeat(n // 1000, 1)
    few, many = local.route(block, 2), local.route(scores, 2)
    assert (many.index.view(-1, 1000, 2) == few.index).all()
    assert (many.weight.view(-1, 1000, 2) == few.weight).all()
    assert torch.equal(many.offsets[1:], few.offsets[1:] * (n // 1000))
    d = torch.randn(1000, 2, generator=g).cuda()
    want = local.route_backward(d, block, few)
    got = local.route_backward(d.repeat(n // 1000, 1), scores, many)
    assert (got.view(-1, 1000, 4) == want).all()


def test_capture_into_a_graph():
    s = _scores(5000, 96, torch.bfloat16, seed=2)
    dw = torch.randn(5000, 4, device="cuda")

    def step():
        r = local.route(s, 4, groups=4, top_groups=2, group_best=2)
        return r.index, r.weight, r.order, r.offsets, local.route_backward(dw, s, r)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for seed in range(4):
        s.copy_(_scores(5000, 96, torch.bfloat16, seed=50 + seed))
        g.replay()
        torch.cuda.synchronize()
        for a, e in zip(out, step()):
            assert torch.equal(a, e)
        torch.cuda.synchronize()


def test_refusals():
    s = _scores(6, 12, torch.float32)
    for bad in (dict(k=0), dict(k=13), dict(k=2, groups=5), dict(k=2, groups=4, top_groups=5),
                dict(k=2, groups=4, top_groups=0), dict(k=2, group_best=3),
                dict(k=2, scale=math.nan), dict(k=2, gate="max"), dict(k=2, bias=s[0, :5])):
        with pytest.raises((ValueError, local.SomError)):
            local.route(s, **bad)
    with pytest.raises(TypeError):
        local.route(s.double(), 2)
    with pytest.raises(TypeError):
        local.route(s, 2, bias=s[0].half())
    with pytest.raises(ValueError):
        local.route(s.t(), 2)
    with pytest.raises(TypeError):
        local.dispatch(torch.zeros(3, 2, device="cuda"), None, 4)
    with pytest.raises(local.SomError):
        local.dispatch(torch.zeros(3, 2, dtype=torch.int32, device="cuda"), None, 0)
    r = local.dispatch(torch.zeros(6, 2, dtype=torch.int32, device="cuda"), None, 12)
    with pytest.raises(ValueError):
        local.route_backward(torch.zeros(6, 2, device="cuda"), s, r)
