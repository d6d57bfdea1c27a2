"""The local models' operators at the ends of their types' ranges, and calls that
have to be refused there."""
import math

import pytest
import torch

import local_oracle as O
from gpu_util import say, torch_cuda
from paper_1905_09598_amd import local

pytestmark = pytest.mark.gpu


def _draw(seed, *shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(dtype).cuda()


@pytest.mark.parametrize("n", [3, 200])
def test_relu_passes_the_gradient_of_a_z_that_rounds_to_zero(n):
    # z = 2^-26 is positive, and 0 in fp16; -2^-26 is not positive
    torch_cuda()
    say("relu next to 0", n)
    half = torch.float16
    x, w = torch.zeros(n, 16, dtype=half, device="cuda"), torch.zeros(8, 16, dtype=half,
                                                                      device="cuda")
    x[:, 0], w[:4, 0], w[4:, 0] = 2.0 ** -12, 2.0 ** -14, -2.0 ** -14
    w[:, 1] = 1.0                       # what dx shows
    y, z = local.linear(x, w, None, "relu", keep=True)
    dx, dw, db = local.linear_backward(torch.ones_like(y), x, w, z, "relu")
    assert (dx[:, 1] == 4).all()
    assert db.tolist() == [n] * 4 + [0] * 4
    assert (dw[:4, 0] > 0).all() and not dw[4:].any()
    # the experts' first layer
    index = torch.zeros(n, 1, dtype=torch.int32, device="cuda")
    r = local.dispatch(index, None, 1)
    w1, w2 = w.unsqueeze(0).contiguous(), torch.ones(1, 8, 8, dtype=half, device="cuda")
    y, kept = local.experts(x, r, w1, None, w2, None, "relu", keep=True)
    g = local.experts_backward(torch.ones_like(y), x, r, w1, None, w2, None, kept, "relu")
    assert (g.x[:, 1] == 4 * 8).all()


@pytest.mark.parametrize("n", [2, 90])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_gradient_of_weights_next_to_zero(dtype, n):
    # weights whose reciprocal is beyond fp32, or denormal, beside ordinary ones, and
    # activations large enough that weight times activation is a normal number
    small = [2.5e-39, 1e-39, 1e-40, 1e-45, 0.0, 2.0 ** -126, 2e-38, 1e-30, 0.25, 1e38, 3.4e38]
    index = torch.arange(n * 3, dtype=torch.int32, device="cuda").view(n, 3) % 4
    weight = torch.tensor([small[s % len(small)] for s in range(n * 3)]).view(n, 3).cuda()
    x = torch.ones(n, 64, dtype=dtype, device="cuda")
    w1 = (1 + _draw(1, 4, 40, 64).abs()).to(dtype)          # z of 64 to some 200
    w2, b2 = _draw(2, 4, 24, 40, dtype=dtype, scale=0.1), _draw(3, 4, 24, dtype=dtype)
    dy = _draw(4, n, 24, dtype=dtype)
    say("weights next to 0", dtype, n)
    ordinary = local.dispatch(index, torch.full_like(weight, 0.5), 4)
    r = local.dispatch(index, weight, 4)
    grads = []
    for route in (r, ordinary):
        kept = local.experts(x, route, w1, None, w2, b2, "gelu", keep=True)[1]
        grads.append(local.experts_backward(dy, x, route, w1, None, w2, b2, kept, "gelu").weight)
    # <dy, answer> does not depend on the weights but by roundings: h to the element type
    # (and an image of it), the result
    e = index.cpu().long()
    h = O.d(x)[:, None, None, :] @ O.d(w1)[e].transpose(2, 3)     # gelu(z) is z here
    a = (O.d(w2)[e] @ h.transpose(2, 3)).squeeze(3) + O.d(b2)[e]
    want = (O.d(dy)[:, None, :] * a).sum(2)
    size = (O.d(dy).abs()[:, None, None, :] @ O.d(w2)[e].abs() @ h.transpose(2, 3)).view(n, 3)
    bound = (2 * O.U[dtype] + 200 * O.V) * size + O.stored(want, dtype)
    for got in grads:
        O.close(got, (want, bound), "dweight")


@pytest.mark.parametrize("hidden", [40, 37])
@pytest.mark.parametrize("n", [6, 150])
def test_small_weights_in_half_precision_keep_their_bits(n, hidden):
    # weights of 1e-4 to 1e-7 and a loss scale that makes up for them: weight times
    # activation is subnormal in fp16 (of few bits, or 0), weight times gradient is not
    say("small weights", n, hidden)
    half, experts, k, inner, outer = torch.float16, 3, 2, 48, 24
    index = torch.arange(n * k, dtype=torch.int32, device="cuda").view(n, k) % experts
    g = torch.Generator().manual_seed(1)
    weight = 10 ** -(4 + 3 * torch.rand(n, k, generator=g)).cuda()
    weight[0, 0] *= -1
    r = local.dispatch(index, weight, experts)
    x = _draw(2, n, inner, dtype=half)
    w1, b1 = _draw(3, experts, hidden, inner, dtype=half, scale=inner ** -0.5), None
    w2 = _draw(4, experts, outer, hidden, dtype=half, scale=hidden ** -0.5)
    dy = _draw(5, n, outer, dtype=half, scale=4000.0)
    dy1 = _draw(6, n, hidden, dtype=half, scale=4000.0)
    kept = local.experts(x, r, w1, b1, w2, None, "gelu", keep=True)[1]
    two = local.experts_backward(dy, x, r, w1, b1, w2, None, kept, "gelu")
    one = local.experts_backward(dy1, x, r, w1, b1, None, None, None)
    tiny, u = O.TINY[half], O.U[half]
    for e in range(experts):
        row, j = (index.cpu() == e).nonzero(as_tuple=True)
        xe, ge = O.d(x)[row], O.d(weight)[row, j].unsqueeze(1)
        (h, herr), _ = O.linear(xe, O.d(w1[e]), None, "gelu", None, half)
        da = ge * O.d(dy)[row]
        want = da.t() @ h
        # scaled, at least half of h: two roundings of its size; dy 2^e may be subnormal
        bound = (2 * da.abs().t() @ herr + tiny * h.abs().sum(0)
                 + (len(row) + 8) * O.V * (da.abs().t() @ h.abs()) + O.stored(want, half))
        O.close(two.w2[e], (want, bound), "dw2")
        da = ge * O.d(dy1)[row]
        want = da.t() @ xe
        bound = ((u + (len(row) + 8) * O.V) * (da.abs().t() @ xe.abs()) + tiny * xe.abs().sum(0)
                 + O.stored(want, half))
        O.close(one.w1[e], (want, bound), "dw1")


@pytest.mark.parametrize("n", [3, 200])
@pytest.mark.parametrize("kind", ["relu", "gelu", "silu"])
def test_gradient_of_a_z_beyond_half_precision(kind, n):
    # z of -80,000 and 80,000: finite sums that fp16 rounds to infinities.  The slopes are
    # 0 and 1, whatever the activation.
    say("large z", kind, n)
    half = torch.float16
    x = torch.zeros(n, 16, dtype=half, device="cuda")
    w = torch.zeros(8, 16, dtype=half, device="cuda")
    x[:, 0], w[:4, 0], w[4:, 0], w[:, 1] = 400.0, 200.0, -200.0, 1.0
    y, z = local.linear(x, w, None, kind, keep=True)
    assert torch.isinf(y[:, :4]).all() and not y[:, 4:].any()
    dx, dw, db = local.linear_backward(torch.ones_like(y), x, w, z, kind)
    assert (dx[:, 1] == 4).all() and (dw[:4, 0] == 400.0 * n if n < 100 else dw[:4, 0] > 0).all()
    assert not dw[4:].any() and db.tolist() == [n] * 4 + [0] * 4
    # infinities of the data stay what they are
    x[0, 0] = math.inf
    z = local.linear(x, w, None, kind, keep=True)[1]
    assert torch.isinf(z[0]).all() and torch.isfinite(z[1:]).all()
    x[0, 0] = math.nan
    assert torch.isnan(local.linear(x, w, None, kind, keep=True)[1][0]).all()


@pytest.mark.parametrize("gate", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts", [12, 16, 64, 640, 4096])
def test_groups_masked_by_the_lowest_value_stay_open(experts, gate):
    # masks of the type's lowest value (finite): two of them add up to -infinity in fp32,
    # which closes no expert.  Row 0: everything masked so; row 1: group 2 is not;
    # row 2: closed (-infinity) but for two masked experts of group 1.
    say("lowest values", experts, gate)
    groups, per = 4, experts // 4
    low = torch.finfo(torch.float32).min
    s = torch.full((3, experts), low, device="cuda")
    s[1, 2 * per:3 * per] = _draw(1, per).cuda()
    s[2] = -math.inf
    s[2, per], s[2, per + 1] = low, low
    bias = None
    if gate == "sigmoid":     # the choice's values are the bias's there: as low
        bias, s = s[0].clone(), torch.zeros_like(s)
        s[2] = -math.inf
        s[2, per], s[2, per + 1] = 0.0, 0.0
    r = local.route(s, 2, bias, gate, groups, 1, 2, renormalise=True)
    index, weight = O.route(s.cpu(), 2, None if bias is None else bias.cpu(), gate, groups, 1, 2)
    assert torch.equal(r.index.cpu().long(), index)
    assert (index >= 0).all()
    assert float((O.d(r.weight) - weight).abs().max()) < 1e-6


def test_the_optimizer_refuses_parameters_that_have_moved():
    # its table holds addresses: a tensor that lies elsewhere by now would not be updated,
    # and what lies at its old place would be
    say("moved parameters")
    p = [_draw(1, 300), _draw(2, 50)]
    opt = local.AdamW(p)
    g = [_draw(3, 300), _draw(4, 50)]
    opt.step(g)
    old, before = p[1].data, p[1].clone()
    p[1].data = old.clone()
    first = p[0].clone()
    with pytest.raises(ValueError):
        opt.step(g)
    assert torch.equal(p[0], first) and torch.equal(old, before) and opt.steps == 1
    p[1].data = old                  # back in its place
    opt.step(g)
    assert opt.steps == 2 and not torch.equal(p[1], before)
    p[0].data = p[0].data[:299]      # shorter
    with pytest.raises(ValueError):
        opt.step(g)


def test_tensors_of_a_graph_are_refused():
    # results carry no graph: a loss on them would leave w without a gradient, silently
    say("graphs")
    x, w, b = _draw(1, 20, 16), _draw(2, 8, 16), _draw(3, 8)
    y = local.linear(x, w, b)
    r = local.route(y, 2)
    w1, dy = _draw(4, 8, 4, 16), _draw(5, 20, 4)
    weight = r.weight.clone()
    calls = {
        "x": (x, lambda: local.linear(x, w, b)), "w": (w, lambda: local.linear(x, w, b)),
        "bias": (b, lambda: local.linear(x, w, b)), "scores": (y, lambda: local.route(y, 2)),
        "balance": (b, lambda: local.route(y, 2, b)), "w1": (w1, lambda: local.experts(x, r, w1)),
        "weight": (weight, lambda: local.dispatch(r.index, weight, 8)),
        "dy": (dy, lambda: local.experts_backward(dy, x, r, w1, None, None, None, None)),
        "dscores": (y, lambda: local.linear_backward(y, x, w)),
        "dweight": (weight, lambda: local.route_backward(weight, y, r)),
    }
    for name, (t, call) in calls.items():
        t.requires_grad_()
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad():
            call()
        t.requires_grad_(False)
        call()
    # the optimizer's parameters may belong to a module
    p = torch.nn.Parameter(_draw(6, 30))
    opt = local.AdamW([p], master=True)
    opt.step([_draw(7, 30)])
    assert not opt.master.requires_grad


@pytest.mark.parametrize("n", [300, 1999, 2000])
def test_example_with_fewer_documents_than_a_batch(n):
    from test_gpu_local_example import _example
    say("example", n)
    seen = []
    module = _example()

    class Counting(module.LocalModels):
        def step(self, x, target):
            seen.append((len(x), len(target)))
            return super().step(x, target)

    module.LocalModels = Counting
    module.run(n=n, steps=4, say=say)
    assert seen == [(n, n)] * 4
