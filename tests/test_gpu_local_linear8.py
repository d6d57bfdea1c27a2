"""Rows brought to 8 bits, to the bit, and products of them against 64 bits: every
element within a bound derived from the roundings and the matrix instruction's own
(layers_oracle)."""
import math

import pytest
import torch

import layers_oracle as O
import paper_1905_09598_amd as som
from gpu_util import say, torch_cuda
from paper_1905_09598_amd import local

pytestmark = pytest.mark.gpu
T = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF = ["bf16", "fp16"]


def _draw(seed, *shape, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(dtype).cuda()


def _held(x):
    b = local.to_blocks(x)
    n, width = x.shape
    count = -(-width // 128)
    assert b.codes.shape == (n, count * 128) and b.scale.shape == (n, -(-count // 4) * 4)
    return b


def _check_blocks(x):
    b = _held(x)
    n, width = x.shape
    count = -(-width // 128)
    value, e = O.blocks(O.d(x))
    powers = b.scale.view(torch.uint8)
    assert torch.equal(powers[:, :count].int() - 127, e)
    assert (powers[:, count:] == 127).all()
    assert (b.codes.view(torch.uint8)[:, width:] == 0).all()
    # in 64 bits: next to fp32's largest number, (2 - 2^-23) 2^127, a code rounds to 256 2^120,
    # which is beyond it
    got = b.codes.double().view(n, count, 128) * powers[:, :count].double().sub(127).exp2().unsqueeze(2)
    got = got.view(n, -1)[:, :width]
    assert torch.equal(torch.isnan(got), torch.isnan(value))
    assert torch.equal(got.nan_to_num(), value.nan_to_num())
    inside = value.abs() < 2.0 ** 128
    assert torch.equal(b.float().double()[inside], value[inside])
    signs = b.codes.view(torch.uint8)[:, :width] >> 7
    fine = ~torch.isnan(value)
    assert torch.equal(signs.bool()[fine], torch.signbit(x)[fine])
    return b


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("n,width", [(1, 1), (3, 7), (2, 127), (5, 128), (4, 129), (33, 500),
                                     (2, 513), (17, 2048), (3, 4545), (1, 70001), (5000, 100)])
def test_blocks_to_the_bit(n, width, dtype):
    torch_cuda()
    say("blocks", n, width, dtype)
    _check_blocks(_draw(n, n, width, dtype=T[dtype], scale=3.0))


@pytest.mark.parametrize("dtype", T)
def test_blocks_of_every_size(dtype):
    """Each value of the type that is positive, in blocks of its neighbours, and magnitudes
    at and next to where the power of two changes."""
    t = T[dtype]
    if t == torch.float32:
        bits = torch.arange(0, 1 << 31, 12347, dtype=torch.int64).int()
    else:
        bits = torch.arange(0, 1 << 15, dtype=torch.int32).to(torch.int16)
    x = bits.view(t)
    x = x[: x.numel() // 128 * 128].view(-1, 128).cuda()
    _check_blocks(x)
    _check_blocks(torch.cat([x.flip(0), -x], 1).contiguous())
    ends = []
    for e in range(-14, 8):
        for v in (1.75, 1.75 + 2.0 ** -7, 1.75 - 2.0 ** -7, 1.0, 2.0 - 2.0 ** -7):
            ends.append(math.ldexp(v, e))
    rows = torch.zeros(len(ends), 128, dtype=t)
    rows[:, 5] = torch.tensor(ends).to(t)
    rows[:, 60] = -0.3 * rows[:, 5]
    _check_blocks(rows.cuda())


def test_blocks_ties_and_numbers_that_are_none():
    # halves of e4m3's steps: 448 keeps the power of two 1
    steps = torch.tensor([448.0, 17.0, 19.0, 21.0, -17.0, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10,
                          2.0 ** -9, 15 * 2.0 ** -10, -0.0, 0.0])
    x = torch.zeros(2, 200)
    x[0, :13], x[1, 140:153] = steps, steps
    _check_blocks(x.cuda())
    x = torch.randn(4, 300, generator=torch.Generator().manual_seed(1))
    x[0, 3], x[1, 130], x[2, 299] = math.nan, math.inf, -math.inf
    x[3, :128] = math.inf
    for t in T.values():
        _check_blocks(x.to(t).cuda())
    zeros = _check_blocks(torch.zeros(3, 256, device="cuda"))
    assert (zeros.scale.view(torch.uint8)[:, :2] == 1).all()


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("offset,gap", [(1, 3), (8, 0), (5, 11)])
def test_blocks_of_strided_rows(offset, gap, dtype):
    wide = torch.full((9, offset + 300 + gap), float("nan"), dtype=T[dtype], device="cuda")
    v = wide[:, offset:offset + 300]
    v.copy_(_draw(1, 9, 300, dtype=T[dtype]))
    _check_blocks(v)
    far = torch.empty((1 << 31) + 8192, dtype=torch.bfloat16, device="cuda")
    v = torch.as_strided(far, (3, 300), (1 << 30, 1))
    v.copy_(_draw(1, 3, 300, dtype=torch.bfloat16))
    _check_blocks(v)


def test_blocks_and_products_of_more_rows_than_one_launch_takes():
    """Four rows of up to 512 values to a workgroup of 256 threads, of which a grid counts
    2^32 - 1: 67,108,860 rows."""
    most = (2 ** 32 - 1) // 256 * 4
    n, ends = most + 1003, [0, 500, most - 300, most, most + 300, most + 1003]
    say("blocks", n)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(n, 3, generator=g, device="cuda", dtype=torch.bfloat16)
    b = local.to_blocks(x)
    w8 = local.to_blocks(_draw(2, 2, 3, dtype=torch.bfloat16))
    bias = _draw(3, 2, dtype=torch.bfloat16)
    for first, last in zip(ends[::2], ends[1::2]):
        part = _check_blocks(x[first:last].contiguous())
        assert torch.equal(b.codes.view(torch.uint8)[first:last], part.codes.view(torch.uint8))
        assert torch.equal(b.scale.view(torch.uint8)[first:last], part.scale.view(torch.uint8))
    del b
    y = local.linear8(x, w8, bias)
    for first, last in zip(ends[::2], ends[1::2]):
        held = local.to_blocks(x[first:last].contiguous())
        O.close(y[first:last], O.linear8(O.d(held.float()), O.d(w8.float()), O.d(bias), "none", None, x.dtype), "y")


def _case(n, inner, outer, dtype, seed=0):
    return (_draw(seed, n, inner, dtype=dtype), _draw(seed + 1, outer, inner, dtype=dtype,
                                                      scale=inner ** -0.5),
            _draw(seed + 2, outer, dtype=dtype), _draw(seed + 3, n, outer, dtype=dtype))


def _check(x, w, b, r, kind):
    w8, x8 = local.to_blocks(w), local.to_blocks(x)
    y = local.linear8(x, w8, b, kind, r)
    want = O.linear8(O.d(x8.float()), O.d(w8.float()), O.d(b), kind, O.d(r), x.dtype)
    O.close(y, want, "y")
    # the same where x comes in 8 bits
    assert torch.equal(local.linear8(x8, w8, b, kind, r, dtype=x.dtype), y)
    # far nearer than the bound as a whole
    u = {torch.bfloat16: 2.0 ** -9, torch.float16: 2.0 ** -12}[x.dtype]
    if y.numel() > 2000 and kind == "none":
        assert float((y.double() - want[0]).norm() / want[0].norm()) < u + 2.0 ** -14
    return y


# one row to several tiles, sizes at, below and beyond blocks, words of scales and tiles
SIZES = [(1, 1, 1), (1, 64, 16), (1, 257, 33), (2, 2048, 129), (5, 10000, 17), (15, 100, 64),
         (16, 640, 1000), (17, 640, 17), (63, 65, 63), (64, 128, 200), (65, 385, 130),
         (100, 8, 300), (129, 520, 136), (256, 256, 256), (300, 1000, 257), (1000, 96, 40),
         (1025, 24, 8), (700, 1537, 121), (1100, 2300, 520)]


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n,inner,outer", SIZES)
def test_products(n, inner, outer, dtype):
    say("linear8", n, inner, outer, dtype)
    x, w, b, r = _case(n, inner, outer, T[dtype], seed=n + inner)
    _check(x, w, b, r, "gelu")
    _check(x, w, None, None, "none")


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("kind", list(local.ACTIVATIONS))
def test_activations_and_absent_parts(kind, dtype):
    for n in (7, 70):
        x, w, b, r = _case(n, 300, 72, T[dtype], seed=5)
        for bb, rr in ((b, r), (None, None), (b, None), (None, r)):
            _check(x, w, bb, rr, kind)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n,inner,outer", [(4000, 128, 4096), (4097, 300, 2048), (200, 9000, 100),
                                           (64, 20001, 64), (2500, 400, 600), (20, 4100, 2000)])
def test_tiles_and_splits(n, inner, outer, dtype):
    x, w, b, r = _case(n, inner, outer, T[dtype], seed=n)
    _check(x, w, b, r, "none")


def _route(n, inner, outer, dtype):
    call = local._Linear8Call(type=local._TYPES[dtype], n=n, inner=inner, outer=outer, ldx=inner)
    route = (local.C.c_int32 * 2)()
    som._check(local.lib().som_linear8_route(local.C.byref(call), route), "som_linear8_route")
    return route[0], route[1]


# every tile, whole and in parts, by the library's own answer; contractions of 1 to 106 blocks,
# so that words of powers begin and end at every place of a slab loop
ROUTES = [(256, False, 4097, 1300, 2048), (256, False, 4097, 640, 2048), (256, False, 1064, 1029, 7750),
          (256, True, 1601, 11700, 2707), (128, False, 637, 128, 8192), (128, False, 2711, 1031, 1481),
          (128, False, 2000, 1537, 3000), (128, True, 827, 13541, 2099), (64, False, 1500, 600, 2500),
          (64, False, 1100, 2300, 520), (64, True, 200, 9000, 100), (64, True, 300, 4545, 300),
          (64, True, 17, 1231, 8), (16, False, 16, 5000, 300), (16, False, 5, 20001, 40)]


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("tile,parts,n,inner,outer", ROUTES)
def test_every_tile_whole_and_in_parts(tile, parts, n, inner, outer, dtype):
    """Rows and blocks whose sizes lie far apart, so that no power of two of another row or
    block passes for their own."""
    say("linear8", tile, parts, n, inner, outer, dtype)
    route = _route(n, inner, outer, T[dtype])
    assert route[0] == tile and (route[1] > 1) == parts, route
    x, w, b, r = _case(n, inner, outer, T[dtype], seed=n)
    g = torch.Generator().manual_seed(3)
    far = 20 if dtype == "bf16" else 3
    for t in (x, w):
        count = -(-inner // 128)
        s = torch.exp2(torch.randint(-far, far, (t.shape[0], count), generator=g).float()).cuda()
        t.mul_(s.repeat_interleave(128, 1)[:, :inner].to(t.dtype))
    _check(x, w, b, r, "none" if dtype == "bf16" else "silu")


@pytest.mark.parametrize("n", [3, 150])
def test_blocks_of_their_own_powers(n):
    """Rows and blocks whose sizes lie far apart: every power of two goes to its own."""
    g = torch.Generator().manual_seed(3)
    x, w, _, _ = _case(n, 1500, 90, torch.bfloat16, seed=1)
    for t in (x, w):
        rows = t.shape[0]
        s = torch.exp2(torch.randint(-20, 20, (rows, 12), generator=g).float()).cuda()
        t.mul_(s.repeat_interleave(128, 1)[:, :1500].to(t.dtype))
    _check(x, w, None, None, "none")


@pytest.mark.parametrize("n", [2, 90])
def test_numbers_that_are_none_stay_in_their_rows(n):
    x, w, b, r = _case(n, 300, 50, torch.bfloat16)
    clean = local.linear8(x, local.to_blocks(w), b)
    x[1, 280] = math.inf
    y = local.linear8(x, local.to_blocks(w), b)
    assert torch.isnan(y[1]).all()
    keep = torch.arange(n, device="cuda") != 1
    assert torch.equal(y[keep], clean[keep])


@pytest.mark.parametrize("n", [3, 200])
@pytest.mark.parametrize("offset,gap", [(0, 8), (1, 3), (5, 11)])
def test_row_strides_and_odd_beginnings(n, offset, gap):
    def strided(seed, cols):
        wide = torch.full((n, offset + cols + gap), float("nan"), dtype=torch.bfloat16, device="cuda")
        v = wide[:, offset:offset + cols]
        v.copy_(_draw(seed, n, cols, dtype=torch.bfloat16))
        return v

    x, r = strided(1, 333), strided(4, 88)
    w, b = _draw(2, 88, 333, dtype=torch.bfloat16), _draw(3, 90, dtype=torch.bfloat16)[2:]
    _check(x, w, b, r, "silu")


def test_no_rows_and_rows_beyond_the_last():
    x, w, b, r = _case(5, 200, 40, torch.bfloat16)
    w8 = local.to_blocks(w)
    assert local.linear8(x[:0], w8, b).shape == (0, 40)
    e8 = local.to_blocks(x[:0])
    assert local.linear8(e8, w8, b, dtype=torch.bfloat16).shape == (0, 40)
    y, whole = local.linear8(x, w8, b), local.linear8(x[:3], w8, b)
    assert torch.equal(y[:3], whole)


def test_the_gradient_of_x_by_the_transpose():
    x, w, _, _ = _case(80, 300, 200, torch.bfloat16)
    dy = _draw(9, 80, 200, dtype=torch.bfloat16)
    t8 = local.to_blocks(w.t().contiguous())
    dx = local.linear8(dy, t8)
    want = O.linear8(O.d(local.to_blocks(dy).float()), O.d(t8.float()), None, "none", None, x.dtype)
    O.close(dx, want, "dx")


def test_streams_graphs_and_repeats():
    x, w, b, r = _case(500, 1000, 200, torch.bfloat16)
    one = x[:1].clone()

    def once():
        w8 = local.to_blocks(w)
        return local.linear8(x, w8, b, "gelu", r), local.linear8(one, w8, b)

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
        x.copy_(_draw(seed, 500, 1000, dtype=torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(held, once()):
            assert torch.equal(u, v)


def test_refusals():
    x, w, b, r = _case(4, 200, 8, torch.bfloat16)
    w8, x8 = local.to_blocks(w), local.to_blocks(x)
    bad = [
        (TypeError, lambda: local.to_blocks(x.double())), (TypeError, lambda: local.to_blocks(x.cpu())),
        (ValueError, lambda: local.to_blocks(x[0])), (ValueError, lambda: local.to_blocks(x[:, :0])),
        (TypeError, lambda: local.linear8(x, w)), (TypeError, lambda: local.linear8(x.float(), w8)),
        (TypeError, lambda: local.linear8(x, w8, dtype=torch.float16)),
        (TypeError, lambda: local.linear8(x8, w8)),
        (TypeError, lambda: local.linear8(x8, w8, dtype=torch.float32)),
        (ValueError, lambda: local.linear8(x[:, :100], w8)),
        (TypeError, lambda: local.linear8(x, w8, b.half())), (ValueError, lambda: local.linear8(x, w8, b[:4])),
        (ValueError, lambda: local.linear8(x, w8, b, residual=r[:2])),
        (ValueError, lambda: local.linear8(x, w8, b, "tanh")),
        (ValueError, lambda: local.linear8(x.clone().requires_grad_(), w8)),
        (TypeError, lambda: local.Blocks(w8.codes.view(torch.uint8), w8.scale, 200)),
        (TypeError, lambda: local.Blocks(w8.codes, w8.scale.float(), 200)),
        (ValueError, lambda: local.Blocks(w8.codes, w8.scale, 300)),
        (ValueError, lambda: local.Blocks(w8.codes[:3], w8.scale, 200)),
        (ValueError, lambda: local.Blocks(w8.codes, w8.scale[:, :2], 200)),
    ]
    for error, call in bad:
        with pytest.raises(error):
            call()
