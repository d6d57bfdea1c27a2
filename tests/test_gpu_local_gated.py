"""The gated layer and its gradients against 64 bits: every element within a bound
derived from the roundings (layers_oracle)."""
import ctypes as C
import math

import pytest
import torch

import layers_oracle as O
import paper_1905_09598_amd as som
from gpu_util import say, torch_cuda
from paper_1905_09598_amd import local

pytestmark = pytest.mark.gpu
T = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _draw(seed, *shape, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(dtype).cuda()


def _case(n, inner, hidden, dtype, seed=0):
    return (_draw(seed, n, inner, dtype=dtype),
            _draw(seed + 1, 2, hidden, inner, dtype=dtype, scale=inner ** -0.5),
            _draw(seed + 2, 2, hidden, dtype=dtype), _draw(seed + 3, n, hidden, dtype=dtype))


def _check(x, w, b, dy, kind):
    y, z = local.gated(x, w, b, kind, keep=True)
    want, wz = O.gated(O.d(x), O.d(w), O.d(b), kind, x.dtype)
    O.close(y, want, "y")
    O.close(z, wz, "z")
    assert torch.equal(local.gated(x, w, b, kind), y)
    dx, dw, db = local.gated_backward(dy, x, w, z, kind)
    g = O.gated_backward(O.d(dy), O.d(x), O.d(w), wz, kind, x.dtype)
    O.close(dx, g["dx"], "dx")
    O.close(dw, g["dw"], "dw")
    O.close(db, g["db"], "db")


# one row to several tiles; sizes at, below and beyond the tiles' halves and their slabs;
# rows that are not whole 16-byte pieces
SIZES = [(1, 1, 1), (1, 64, 16), (1, 257, 33), (2, 2048, 129), (15, 100, 64), (16, 64, 1000),
         (17, 640, 17), (63, 65, 31), (64, 72, 32), (65, 33, 65), (100, 8, 300), (129, 520, 72),
         (256, 256, 128), (300, 1000, 129), (1000, 96, 40), (1025, 24, 8), (700, 1537, 61),
         (2000, 300, 501)]


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("n,inner,hidden", SIZES)
def test_layer_and_gradients(n, inner, hidden, dtype):
    torch_cuda()
    say("gated", n, inner, hidden, dtype)
    _check(*_case(n, inner, hidden, T[dtype], seed=n + inner), kind="silu")


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("n", [5, 70])
@pytest.mark.parametrize("kind", list(local.ACTIVATIONS))
def test_activations_and_absent_parts(kind, n, dtype):
    x, w, b, dy = _case(n, 136, 72, T[dtype], seed=5)
    _check(x, w, b, dy, kind)
    _check(x, w, None, dy, kind)
    z = local.gated(x, w, None, kind, keep=True)[1]
    assert local.gated_backward(dy, x, w, z, kind, bias=False)[2] is None


def _tiles(call, backward):
    tiles = (C.c_int32 * 2)()
    som._check(local.lib().som_gated_route(C.byref(call), backward, tiles), "som_gated_route")
    return list(tiles)


@pytest.mark.parametrize("dtype", T)
def test_every_tile(dtype):
    """Sizes at which the choice takes several tiles, in whole 16-byte pieces and not, with
    long contractions that are split."""
    t, seen = T[dtype], set()
    for n, inner, hidden in [(4096, 64, 2048), (3000, 64, 500), (200, 128, 96), (300, 8000, 100),
                             (3001, 61, 2051), (100, 67, 33), (70, 4000, 24), (70, 4001, 24)]:
        x, w, b, dy = _case(n, inner, hidden, t, seed=n)
        call = local._gated_call(x, w, "gelu")
        seen.add(_tiles(call, 0)[0])
        _check(x, w, b, dy, "gelu")
    say("tiles of", dtype, sorted(seen))
    assert len(seen) >= 3


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("n", [3, 200])
@pytest.mark.parametrize("offset,gap", [(0, 8), (1, 3), (8, 0), (5, 11)])
def test_row_strides_and_odd_beginnings(n, offset, gap, dtype):
    inner, hidden = 120, 44
    dtype = T[dtype]

    def strided(seed, cols):
        wide = torch.full((n, offset + cols + gap), float("nan"), dtype=dtype, device="cuda")
        v = wide[:, offset:offset + cols]
        v.copy_(_draw(seed, n, cols, dtype=dtype))
        return v

    x, dy = strided(1, inner), strided(4, hidden)
    room = torch.empty(2 * hidden * inner + offset, dtype=dtype, device="cuda")
    w = room[offset:].view(2, hidden, inner)
    w.copy_(_draw(2, 2, hidden, inner, dtype=dtype, scale=inner ** -0.5))
    b = _draw(3, 2 * hidden + offset, dtype=dtype)[offset:].view(2, hidden)
    _check(x, w, b, dy, "gelu")


def _scaled(n, inner, hidden, x, w, u, v, dy, seed=1):
    """fp16 inputs of these sizes: x and w of normal values, biases about u and v."""
    t = torch.float16
    b = torch.cat([_draw(seed + 2, 1, hidden, dtype=torch.float32, scale=u),
                   v * (1 + 0.2 * _draw(seed + 4, 1, hidden, dtype=torch.float32))]).to(t)
    return (_draw(seed, n, inner, dtype=t, scale=x), _draw(seed + 1, 2, hidden, inner, dtype=t, scale=w),
            b, _draw(seed + 3, n, hidden, dtype=t, scale=dy))


def _check_powers(x, w, b, dy, kind):
    z = local.gated(x, w, b, kind, keep=True)[1]
    wz = O.gated(O.d(x), O.d(w), O.d(b), kind, x.dtype)[1]
    got = dict(zip(("dx", "dw", "db"), local.gated_backward(dy, x, w, z, kind)))
    g = O.gated_backward(O.d(dy), O.d(x), O.d(w), wz, kind, x.dtype, powers=True)
    for name, t in got.items():
        value, bound = g[name]
        ordinary = value.abs() < 65000      # beyond, fp16 rounds to infinity
        assert name == "db" or ordinary.all(), name
        O.close(t[ordinary], (value[ordinary], bound[ordinary]), name)


# sizes of x, w, u, v and dy: dy v of 10^6 and more, whose products with w and x are ordinary
# numbers; dy v of 10^-7 and less, whose products with large x or w are; and dy v between
@pytest.mark.parametrize("kind", ["silu", "gelu", "none"])
@pytest.mark.parametrize("n,inner,hidden", [(1, 40, 24), (70, 129, 33), (600, 520, 264), (5000, 64, 500)])
@pytest.mark.parametrize("x,w,u,v,dy", [(3e-5, 1e-4, 1.0, 20000.0, 100.0), (1e-6, 1e-6, 1.0, 3e4, 2e3),
                                        (2000.0, 1e-4, 0.5, 0.01, 1e-5), (0.001, 50.0, 0.5, 0.02, 3e-6),
                                        (300.0, 0.003, 0.5, 1.0, 2e-4), (1.0, 0.05, 1.0, 1.0, 1.0)])
def test_gradients_of_every_size_in_fp16(x, w, u, v, dy, n, inner, hidden, kind):
    say("gated powers", x, w, v, dy, n, inner, hidden, kind)
    _check_powers(*_scaled(n, inner, hidden, x, w, u, v, dy), kind)


def test_fp16_gradients_without_a_largest_number():
    """All zeros; numbers that are none, which leave the others' power alone."""
    x, w, b, dy = _scaled(90, 72, 40, 1.0, 0.1, 1.0, 1.0, 1e-6)
    z = local.gated(x, w, b, keep=True)[1]
    for t in local.gated_backward(torch.zeros_like(dy), x, w, z):
        assert float(t.abs().max()) == 0
    clean = local.gated_backward(dy, x, w, z)
    dy[5, 3], dy[6, 4] = math.inf, math.nan
    dx, dw, db = local.gated_backward(dy, x, w, z)
    keep = torch.tensor([i not in (5, 6) for i in range(90)], device="cuda")
    assert torch.equal(dx[keep], clean[0][keep]) and not torch.isfinite(dx[5:7]).any()
    rows = torch.tensor([i not in (3, 4) for i in range(40)], device="cuda")
    assert torch.equal(dw[:, rows], clean[1][:, rows]) and torch.equal(db[:, rows], clean[2][:, rows])


def test_fp16_powers_of_replays_are_their_own():
    """A captured gradient takes the power of two that each replay's values ask for."""
    x, w, b, dy = _scaled(300, 256, 96, 0.001, 0.01, 1.0, 100.0, 1.0)
    z = local.gated(x, w, b, keep=True)[1]
    first = dy.clone()
    local.gated_backward(dy, x, w, z)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = local.gated_backward(dy, x, w, z)
    for size in (1.0, 2.0 ** 10, 2.0 ** -16, 1.0, 2.0 ** -18, 2.0 ** 9):
        dy.copy_(first * size)
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(got, local.gated_backward(dy, x, w, z)):
            assert torch.equal(a, c)
        g = O.gated_backward(O.d(dy), O.d(x), O.d(w), O.gated(O.d(x), O.d(w), O.d(b), "silu", x.dtype)[1], "silu",
                             x.dtype, powers=True)
        O.close(got[1], g["dw"], "dw")


@pytest.mark.parametrize("dtype", T)
def test_many_rows_of_few_columns(dtype):
    _check(*_case(20000, 16, 5, T[dtype], seed=3), kind="gelu")


def test_no_rows():
    x, w, b, dy = _case(0, 40, 24, torch.bfloat16)
    y, z = local.gated(x, w, b, keep=True)
    assert y.shape == (0, 24) and z.shape == (0, 2, 24)
    dx, dw, db = local.gated_backward(dy, x, w, z)
    assert dx.shape == (0, 40) and float(dw.abs().max()) == 0 and float(db.abs().max()) == 0


@pytest.mark.parametrize("n", [2, 80])
def test_numbers_that_are_none(n):
    x, w, b, dy = _case(n, 64, 32, torch.float32)
    x[1, 3] = math.nan
    y, z = local.gated(x, w, b, keep=True)
    bad = torch.zeros(n, dtype=torch.bool, device="cuda")
    bad[1] = True
    assert torch.equal(torch.isnan(y).all(1), bad) and torch.equal(torch.isnan(y).any(1), bad)
    # far from 0 the activation's slope is 0 or 1, not a NaN
    x[1], w[0] = 1e15, 1e15
    x[1, ::2] = -3e14
    y, z = local.gated(x, w, b, keep=True)
    assert torch.isfinite(z).all()
    assert torch.isfinite(local.gated_backward(dy, x, w, z)[2]).all()


def test_halves_are_the_two_products():
    """y of the two matrices is the product of linear's results, in either order where
    there is no activation."""
    x, w, b, _ = _case(300, 128, 64, torch.float32, seed=8)
    u, v = local.linear(x, w[0].contiguous(), b[0].contiguous(), "gelu"), local.linear(
        x, w[1].contiguous(), b[1].contiguous())
    y = local.gated(x, w, b, "gelu")
    assert torch.allclose(y, u * v, rtol=1e-4, atol=1e-5)
    swapped = local.gated(x, w.flip(0).contiguous(), b.flip(0).contiguous(), "none")
    assert torch.equal(swapped, local.gated(x, w, b, "none"))


def test_streams_graphs_and_repeats():
    x, w, b, dy = _case(500, 512, 200, torch.bfloat16)

    def once():
        y, z = local.gated(x, w, b, keep=True)
        return (y, z, *local.gated_backward(dy, x, w, z))

    want = once()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = once()
    side.synchronize()
    for u, v in zip(want, got):
        assert torch.equal(u, v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = once()
    for seed in (5, 6, 7):
        x.copy_(_draw(seed, 500, 512, dtype=torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(held, once()):
            assert torch.equal(u, v)


def test_refusals():
    x, w, b, dy = _case(4, 16, 8, torch.float32)
    _, z = local.gated(x, w, keep=True)
    bad = [
        (TypeError, lambda: local.gated(x.double(), w)), (TypeError, lambda: local.gated(x.cpu(), w)),
        (TypeError, lambda: local.gated(x, w.bfloat16())), (ValueError, lambda: local.gated(x, w[0])),
        (ValueError, lambda: local.gated(x, w[:1])), (ValueError, lambda: local.gated(x, w[:, :0])),
        (ValueError, lambda: local.gated(x[:, :8], w)), (ValueError, lambda: local.gated(x, w, b[0])),
        (ValueError, lambda: local.gated(x, w.transpose(1, 2).contiguous().transpose(1, 2))),
        (ValueError, lambda: local.gated(x, w, b, "tanh")),
        (ValueError, lambda: local.gated(x.clone().requires_grad_(), w)),
        (TypeError, lambda: local.gated_backward(dy, x, w, None)),
        (TypeError, lambda: local.gated_backward(dy, x, w, z.bfloat16())),
        (ValueError, lambda: local.gated_backward(dy, x, w, z[:3])),
        (ValueError, lambda: local.gated_backward(dy[:, :4], x, w, z)),
    ]
    for error, call in bad:
        with pytest.raises(error):
            call()
