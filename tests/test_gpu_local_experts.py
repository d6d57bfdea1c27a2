"""The routed experts' products, the join of their answers and the gradients
against 64 bits, product by product within derived bounds."""
import pytest
import torch

import local_oracle as O
from gpu_util import say, torch_cuda
from paper_1905_09598_amd import local

pytestmark = pytest.mark.gpu
T = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _draw(seed, *shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(dtype).cuda()


def _index(n, k, experts, seed, absent=0.1, popular=0.0):
    g = torch.Generator().manual_seed(seed)
    index = torch.randint(0, experts, (n, k), generator=g, dtype=torch.int32)
    if popular:
        index[torch.rand(n, k, generator=g) < popular] = experts // 2
    index[torch.rand(n, k, generator=g) < absent] = -1
    return index.cuda()


def _case(n, k, experts, inner, hidden, outer, dtype, seed=0, **how):
    index = _index(n, k, experts, seed, **how)
    weight = _draw(seed + 1, n, k).softmax(1)
    return (_draw(seed + 2, n, inner, dtype=dtype), local.dispatch(index, weight, experts),
            _draw(seed + 3, experts, hidden, inner, dtype=dtype, scale=inner ** -0.5),
            _draw(seed + 4, experts, hidden, dtype=dtype),
            _draw(seed + 5, experts, outer, hidden, dtype=dtype, scale=hidden ** -0.5),
            _draw(seed + 6, experts, outer, dtype=dtype), _draw(seed + 7, n, outer, dtype=dtype))


def _forward(x, r, w1, b1, w2, b2, kind, residual, dtype):
    """Value and bound of the joined answers, and what the gradient needs."""
    n, k = r.index.shape
    index, weight = r.index.cpu().long(), O.d(r.weight)
    outer = (w1 if w2 is None else w2).shape[1]
    y, err = torch.zeros(n, outer).double(), torch.zeros(n, outer).double()
    if residual is not None:
        y += O.d(residual)
        err += (k + 4) * O.V * O.d(residual).abs()
    kept = []
    for e in range(r.experts):
        row, j = (index == e).nonzero(as_tuple=True)
        if not row.numel():
            continue
        xe, g = O.d(x)[row], weight[row, j].unsqueeze(1)
        (h, herr), (z, zerr) = O.linear(xe, O.d(w1[e]), None if b1 is None else O.d(b1[e]),
                                        kind if w2 is not None else "none", None, dtype)
        if w2 is None:
            a, aerr = h, herr
        else:
            (a, aerr), _ = O.linear(h, O.d(w2[e]), None if b2 is None else O.d(b2[e]), "none",
                                    None, dtype)
            w2a = O.d(w2[e]).abs()
            aerr = aerr + (1 + (h.shape[1] + 8) * O.V) * (herr @ w2a.t())
        y.index_add_(0, row, g * a)
        err.index_add_(0, row, g.abs() * (aerr + (k + 4) * O.V * a.abs()))
        kept.append((e, row, j, xe, g, h, herr, z, zerr, a, aerr))
    return (y, err + O.stored(y, dtype)), kept


def _check(x, r, w1, b1, w2, b2, residual, kind="gelu"):
    dtype = x.dtype
    n, k = r.index.shape
    y, held = local.experts(x, r, w1, b1, w2, b2, kind, residual, keep=True)
    want, kept = _forward(x, r, w1, b1, w2, b2, kind, residual, dtype)
    O.close(y, want, "y")
    assert torch.equal(y, local.experts(x, r, w1, b1, w2, b2, kind, residual))
    dy = _draw(99, *y.shape, dtype=dtype)
    got = local.experts_backward(dy, x, r, w1, b1, w2, b2, held, kind)
    dyc = O.d(dy)
    zero = lambda t: [torch.zeros(t.shape).double(), torch.zeros(t.shape).double()]  # noqa: E731
    dx, dweight, dw1, db1 = zero(x), zero(r.weight), zero(w1), zero(w1[:, :, 0])
    dw2, db2 = (zero(w2), zero(w2[:, :, 0])) if w2 is not None else (None, None)
    for e, row, j, xe, g, h, herr, z, zerr, a, aerr in kept:
        d = dyc[row]
        dot = (d * a).sum(1)
        dweight[0][row, j] = dot
        dweight[1][row, j] = ((d.abs() * aerr).sum(1)
                              + (d.shape[1] + 8) * O.V * (d * a).abs().sum(1)
                              + O.stored(dot, dtype))
        da = g * d
        daerr = O.stored(da, dtype) + 2 * O.V * da.abs()
        if w2 is not None:
            full = da.abs() + daerr
            dw2[0][e] = da.t() @ h
            dw2[1][e] = (daerr.t() @ h.abs() + full.t() @ herr
                         + (len(row) + 8) * O.V * (full.t() @ (h.abs() + herr))
                         + O.stored(dw2[0][e], dtype))
            db2[0][e] = da.sum(0)
            db2[1][e] = (daerr.sum(0) + (len(row) + 8) * O.V * full.sum(0)
                         + O.stored(db2[0][e], dtype))
            w = O.d(w2[e])
            dh = da @ w
            dherr = daerr @ w.abs() + (w.shape[0] + 8) * O.V * (full @ w.abs())
            b = O.linear_backward(dh, xe, O.d(w1[e]), z, zerr, kind, dtype, dherr, True)
        else:
            b = O.linear_backward(da, xe, O.d(w1[e]), z, zerr, "none", dtype, daerr, False)
        dx[0].index_add_(0, row, b["dx"][0])
        dx[1].index_add_(0, row, b["dx"][1] + (k + 4) * O.V * b["dx"][0].abs())
        (dw1[0][e], dw1[1][e]), (db1[0][e], db1[1][e]) = b["dw"], b["db"]
    dx[1] += O.stored(dx[0], dtype)
    tiny = O.TINY[dtype]
    for name, val in (("x", dx), ("weight", dweight), ("w1", dw1), ("b1", db1), ("w2", dw2),
                      ("b2", db2)):
        if val is None or (name == "b1" and b1 is None) or (name == "b2" and b2 is None):
            assert getattr(got, name) is None
        else:
            O.close(getattr(got, name), (val[0], val[1] + tiny), "d" + name)


SIZES = [(1, 1, 1, 8, 8, 8), (1, 4, 64, 200, 72, 200), (5, 2, 3, 33, 17, 21),
         (40, 2, 8, 64, 64, 64), (100, 3, 70, 96, 40, 56), (300, 2, 5, 130, 129, 66),
         (600, 1, 4, 72, 264, 40), (900, 2, 3, 256, 136, 304)]


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("n,k,experts,inner,hidden,outer", SIZES)
def test_experts_and_gradients(n, k, experts, inner, hidden, outer, dtype):
    torch_cuda()
    say("experts", n, k, experts, inner, hidden, outer, dtype)
    x, r, w1, b1, w2, b2, res = _case(n, k, experts, inner, hidden, outer, T[dtype], seed=n)
    _check(x, r, w1, b1, w2, b2, res)


@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
def test_activations(kind):
    x, r, w1, b1, w2, b2, res = _case(90, 2, 6, 48, 80, 56, torch.float16, seed=4)
    _check(x, r, w1, b1, w2, b2, res, kind)


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("n", [2, 150])
def test_local_linear_maps_and_absent_parts(n, dtype):
    x, r, w1, b1, w2, b2, _ = _case(n, 2, 5, 64, 40, 48, T[dtype], seed=9)
    res = _draw(5, n, 40, dtype=T[dtype])
    _check(x, r, w1, b1, None, None, res)
    _check(x, r, w1, None, None, None, None)
    _check(x, r, w1, None, w2, None, None)


def test_popular_experts_and_experts_without_documents():
    x, r, w1, b1, w2, b2, res = _case(700, 2, 40, 64, 72, 64, torch.bfloat16, seed=3,
                                      popular=0.8)
    index = torch.where(r.index % 7 == 3, -1, r.index).int()
    r = local.dispatch(index, r.weight, 40)
    assert int((r.load == 0).sum()) >= 5 and int(r.load.max()) > 700
    _check(x, r, w1, b1, w2, b2, res)


def test_nothing_routed():
    x, _, w1, b1, w2, b2, res = _case(20, 2, 4, 32, 16, 24, torch.float32)
    r = local.dispatch(torch.full((20, 2), -1, dtype=torch.int32, device="cuda"),
                       torch.zeros(20, 2, device="cuda"), 4)
    _check(x, r, w1, b1, w2, b2, res)
    y = local.experts(x, r, w1, b1, w2, b2)
    assert not y.any()


def test_no_documents():
    x, _, w1, b1, w2, b2, _ = _case(4, 2, 4, 32, 16, 24, torch.bfloat16)
    r = local.route(torch.zeros(0, 4, device="cuda"), 2)
    y, held = local.experts(x[:0], r, w1, b1, w2, b2, "gelu", keep=True)
    assert y.shape == (0, 24)
    g = local.experts_backward(y, x[:0], r, w1, b1, w2, b2, held)
    assert g.x.shape == (0, 32) and g.weight.shape == (0, 2)
    assert not g.w1.any() and not g.b1.any() and not g.w2.any() and not g.b2.any()


def test_spoilt_rows_show():
    # a NaN score: the document's weights, and so its answer, are NaN, no other's
    x, _, w1, b1, w2, b2, res = _case(50, 2, 8, 32, 16, 32, torch.float32)
    s = _draw(1, 50, 8)
    clean = local.experts(x, local.route(s, 2), w1, b1, w2, b2, residual=res)
    s[7, 3] = float("nan")
    y = local.experts(x, local.route(s, 2), w1, b1, w2, b2, residual=res)
    assert torch.isnan(y[7]).all()
    keep = torch.arange(50) != 7
    assert torch.equal(y[keep], clean[keep])


def test_document_twice_at_one_expert_and_strided_documents():
    wide = torch.full((60, 100), float("nan"), dtype=torch.bfloat16, device="cuda")
    x = wide[:, 8:72]
    x.copy_(_draw(1, 60, 64, dtype=torch.bfloat16))
    index = _index(60, 3, 2, 5, absent=0.0)
    r = local.dispatch(index, _draw(2, 60, 3).softmax(1), 2)
    _, _, w1, b1, w2, b2, res = _case(60, 3, 2, 64, 48, 40, torch.bfloat16)
    _check(x, r, w1, b1, w2, b2, res)


def test_gradients_are_the_slopes_of_the_loss():
    x, r, w1, b1, w2, b2, res = _case(12, 2, 4, 10, 9, 8, torch.float32, seed=2)
    dy = _draw(50, 12, 8)
    held = local.experts(x, r, w1, b1, w2, b2, "silu", res, keep=True)[1]
    g = local.experts_backward(dy, x, r, w1, b1, w2, b2, held, "silu")
    args = [O.d(t) for t in (x, r.weight, w1, b1, w2, b2)]
    for i, grad in enumerate((g.x, g.weight, g.w1, g.b1, g.w2, g.b2)):
        v = O.d(_draw(60 + i, *grad.shape))

        def loss(t):
            a = list(args)
            a[i] = a[i] + t * v
            y = O.experts(a[0], r.index.cpu(), a[1], a[2], a[3], a[4], a[5], "silu", O.d(res))
            return float((y * O.d(dy)).sum())

        slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
        assert abs(float((O.d(grad) * v).sum()) - slope) <= 1e-5 * (1 + abs(slope)), i


def test_runs_are_equal_bit_for_bit():
    x, r, w1, b1, w2, b2, res = _case(500, 2, 30, 128, 64, 128, torch.bfloat16, seed=8)
    dy = _draw(3, 500, 128, dtype=torch.bfloat16)
    runs = []
    for _ in range(3):
        y, held = local.experts(x, r, w1, b1, w2, b2, "gelu", res, keep=True)
        g = local.experts_backward(dy, x, r, w1, b1, w2, b2, held, "gelu")
        runs.append((y, g.x, g.weight, g.w1, g.b1, g.w2, g.b2))
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))


def test_refusals():
    x, r, w1, b1, w2, b2, res = _case(10, 2, 4, 32, 16, 24, torch.float32)
    with pytest.raises(ValueError):
        local.experts(x[:9], r, w1, b1, w2, b2)
    with pytest.raises(ValueError):
        local.experts(x, r, w1[:3], b1, w2, b2)
    with pytest.raises(ValueError):
        local.experts(x, r, w1, b1, w2[:, :, :15], b2)
    with pytest.raises(ValueError):
        local.experts(x, r, w1, b1, None, b2)
    with pytest.raises(TypeError):
        local.experts(x, r, w1.half(), b1, w2, b2)
    with pytest.raises(ValueError):
        local.experts(x, r, w1, b1, w2, b2, residual=res[:, :5])
    with pytest.raises(TypeError):
        local.experts(x.cpu(), r, w1, b1, w2, b2)
