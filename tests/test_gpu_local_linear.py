"""The product with its epilogue and its gradients against 64 bits: every
element within a bound derived from the roundings (local_oracle)."""
import pytest
import torch

import local_oracle as O
import paper_1905_09598_amd as som
from gpu_util import say, torch_cuda
from paper_1905_09598_amd import local

pytestmark = pytest.mark.gpu
T = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _draw(seed, *shape, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(dtype).cuda()


def _case(n, inner, outer, dtype, seed=0):
    return (_draw(seed, n, inner, dtype=dtype),
            _draw(seed + 1, outer, inner, dtype=dtype, scale=inner ** -0.5),
            _draw(seed + 2, outer, dtype=dtype), _draw(seed + 3, n, outer, dtype=dtype),
            _draw(seed + 4, n, outer, dtype=dtype))


def _check(x, w, b, r, dy, kind):
    dtype = x.dtype
    y, z = local.linear(x, w, b, kind, r, keep=True)
    want, wz = O.linear(O.d(x), O.d(w), O.d(b), kind, O.d(r), dtype)
    O.close(y, want, "y")
    if kind != "none":
        O.close(z, wz, "z")
    dx, dw, db = local.linear_backward(dy, x, w, z, kind)
    g = O.linear_backward(O.d(dy), O.d(x), O.d(w), wz[0], wz[1], kind, dtype)
    O.close(dx, g["dx"], "dx")
    O.close(dw, g["dw"], "dw")
    O.close(db, g["db"], "db")


# one row to several tiles; sizes at, below and beyond the tiles and their slabs;
# rows that are not whole 16-byte pieces
SIZES = [(1, 1, 1), (1, 64, 16), (1, 257, 33), (2, 2048, 129), (15, 100, 64), (16, 64, 1000),
         (17, 640, 17), (63, 65, 63), (64, 72, 200), (65, 33, 130), (100, 8, 300),
         (129, 520, 136), (256, 256, 256), (300, 1000, 257), (1000, 96, 40), (1025, 24, 8),
         (700, 1537, 121)]


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("n,inner,outer", SIZES)
def test_product_and_gradients(n, inner, outer, dtype):
    torch_cuda()
    say("linear", n, inner, outer, dtype)
    _check(*_case(n, inner, outer, T[dtype], seed=n + inner), kind="gelu")


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("kind", list(local.ACTIVATIONS))
def test_activations_and_absent_parts(kind, dtype):
    x, w, b, r, dy = _case(70, 136, 72, T[dtype], seed=5)
    _check(x, w, b, r, dy, kind)
    for bb, rr in ((None, None), (b, None), (None, r)):
        y = local.linear(x, w, bb, kind, rr)
        O.close(y, O.linear(O.d(x), O.d(w), O.d(bb), kind, O.d(rr), x.dtype)[0], (kind,))
    z = local.linear(x, w, None, kind, keep=True)[1]
    assert local.linear_backward(dy, x, w, z, kind, bias=False)[2] is None


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("n", [3, 200])
@pytest.mark.parametrize("offset,gap", [(0, 8), (1, 3), (8, 0), (5, 11)])
def test_row_strides_and_odd_beginnings(n, offset, gap, dtype):
    inner, outer = 120, 88
    dtype = T[dtype]

    def strided(seed, cols):
        wide = torch.full((n, offset + cols + gap), float("nan"), dtype=dtype, device="cuda")
        v = wide[:, offset:offset + cols]
        v.copy_(_draw(seed, n, cols, dtype=dtype))
        return v

    x, r, dy = strided(1, inner), strided(2, outer), strided(3, outer)
    _, w, b, _, _ = _case(n, inner, outer, dtype)
    w1 = torch.cat([w.flatten()[:1], w.flatten()])[1:].view(outer, inner)  # off 16 bytes
    _check(x, w, b, r, dy, "silu")
    _check(x, w1, b, r, dy, "none")


@pytest.mark.parametrize("dtype", T)
def test_no_rows(dtype):
    x, w, b, r, dy = _case(0, 40, 24, T[dtype])
    y, z = local.linear(x, w, b, "gelu", r, keep=True)
    assert y.shape == (0, 24) and z.shape == (0, 24)
    dx, dw, db = local.linear_backward(dy, x, w, z, "gelu")
    assert dx.shape == (0, 40) and not dw.any() and not db.any()


def test_rows_beyond_32_bits():
    # three rows 2.2 GB apart: byte offsets of the last pass 2^32
    ld, inner, outer = 1_100_000_000, 192, 80
    base = torch.empty(2 * ld + inner, dtype=torch.bfloat16, device="cuda")
    x = base.as_strided((3, inner), (ld, 1))
    x.copy_(_draw(1, 3, inner, dtype=torch.bfloat16))
    _, w, b, _, dy = _case(3, inner, outer, torch.bfloat16)
    _check(x, w, b, None, dy, "none")
    big = base.as_strided((2 * ld // 1_000_000, inner), (1_000_000, 1))  # the tiles' path
    big.copy_(_draw(2, big.shape[0], inner, dtype=torch.bfloat16))
    dy = _draw(3, big.shape[0], outer, dtype=torch.bfloat16)
    _check(big, w, b, None, dy, "relu")


def test_sums_of_many_rows():
    # small whole numbers: every partial sum is exact, whatever the order
    n = 8_500_000
    g = torch.Generator(device="cuda").manual_seed(9)
    x, dy = (torch.randint(-1, 2, (n, 8), generator=g, device="cuda").to(torch.bfloat16)
             for _ in range(2))
    w = _draw(1, 8, 8, dtype=torch.bfloat16)
    _, dw, db = local.linear_backward(dy, x, w)
    assert torch.equal(db, dy.double().sum(0).to(torch.bfloat16))
    assert torch.equal(dw, (dy.double().t() @ x.double()).to(torch.bfloat16))


def test_long_contraction_is_split_and_joined():
    # few tiles, long sums: the contraction is split and joined in a fixed order
    for n, inner, outer in ((40, 20000, 24), (70, 9001, 30)):
        x, w, b, r, dy = _case(n, inner, outer, torch.float32, seed=7)
        _check(x, w, b, r, dy, "silu")
        again = [local.linear(x, w, b, "silu", r) for _ in range(3)]
        assert all(torch.equal(again[0], a) for a in again)


def test_gradients_are_the_slopes_of_the_loss():
    # <gradient, direction> against the difference of the 64-bit loss
    for kind in ("gelu", "silu"):
        x, w, b, r, dy = _case(33, 50, 29, torch.float32, seed=11)
        z = local.linear(x, w, b, kind, r, keep=True)[1]
        grads = local.linear_backward(dy, x, w, z, kind)
        h = 1e-5
        for i, (g, at) in enumerate(zip(grads, (x, w, b))):
            v = O.d(_draw(20 + i, *at.shape, dtype=torch.float32))

            def loss(t):
                args = [O.d(x), O.d(w), O.d(b)]
                args[i] = args[i] + t * v
                zz = args[0] @ args[1].t() + args[2]
                return float((O.act(zz, kind) * O.d(dy)).sum())

            slope = (loss(h) - loss(-h)) / (2 * h)
            # fp32 gradient: each element within (K + 24) v of sums of magnitudes ~ 50
            assert abs(float((O.d(g) * v).sum()) - slope) <= 1e-4 * (1 + abs(slope)), (kind, i)


@pytest.mark.parametrize("n", [4, 300])
def test_infinities_and_nan_stay_where_they_belong(n):
    x, w, b, r, _ = _case(n, 128, 96, torch.bfloat16, seed=3)
    y0 = local.linear(x, w, b, "none", r)
    x[2, 7] = float("nan")
    x[0, 3] = float("inf")
    y = local.linear(x, w, b, "none", r)
    assert torch.isnan(y[2]).all() and not torch.isfinite(y[0]).any()
    keep = torch.ones(n, dtype=torch.bool)
    keep[[0, 2]] = False
    assert torch.equal(y[keep], y0[keep])


def test_another_stream():
    x, w, b, r, dy = _case(500, 256, 264, torch.float16, seed=2)
    ref = local.linear(x, w, b, "gelu", r)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a = x * 2
        y = local.linear(a, w, b, "gelu", r)
        z = local.linear(x, w, b, "gelu", r)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(z, ref)
    assert torch.equal(y, local.linear(x * 2, w, b, "gelu", r))


def test_capture_into_a_graph():
    x, w, b, r, dy = _case(130, 300, 72, torch.bfloat16, seed=4)

    def step():
        y, z = local.linear(x, w, b, "gelu", r, keep=True)
        return (y, *local.linear_backward(dy, x, w, z, "gelu"))

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for seed in range(4):
        x.copy_(_draw(40 + seed, 130, 300, dtype=torch.bfloat16))
        g.replay()
        torch.cuda.synchronize()
        for a, e in zip(out, step()):
            assert torch.equal(a, e)
        torch.cuda.synchronize()


def test_refusals():
    x, w, b, r, dy = _case(8, 32, 16, torch.float32)
    with pytest.raises(TypeError):
        local.linear(x.double(), w.double())
    with pytest.raises(TypeError):
        local.linear(x.cpu(), w)
    with pytest.raises(TypeError):
        local.linear(x, w.half())
    with pytest.raises(ValueError):
        local.linear(x, w[:, :31])
    with pytest.raises(ValueError):
        local.linear(x, w.t().contiguous().t())
    with pytest.raises(ValueError):
        local.linear(x.t(), w)
    with pytest.raises(ValueError):
        local.linear(x, w, b[:15])
    with pytest.raises(ValueError):
        local.linear(x, w, b, "tanh")
    with pytest.raises(ValueError):
        local.linear(x, w, b, residual=r[:7])
    with pytest.raises(ValueError):
        local.linear(x[:1].expand(8, 32), w)           # rows on top of each other
    with pytest.raises(ValueError):
        local.linear_backward(dy, x, w, None, "gelu")  # needs z
    with pytest.raises(ValueError):
        local.linear_backward(dy[:, :8], x, w)
    # the C entry: a workspace that is too small, and arrays past their allocation
    x, w, y = (torch.zeros(*s, device="cuda") for s in ((40, 20000), (24, 20000), (40, 24)))
    call = local._dense_call(x, w, "none")     # a contraction that is split
    call.y = y.data_ptr()
    assert som.STATUS[local.lib().som_linear(call)] == "SOM_E_ARG"
    call.n = 1 << 38
    assert som.STATUS[local.lib().som_linear(call)] == "SOM_E_ARG"
