"""Every tile that a product can run in, in every mode, against 64 bits: sizes off
the tiles and their slabs, contractions of several slabs, and the tile asserted by the
library's own answer, so that a change of the plan shows here."""
import ctypes as C

import pytest
import torch

import test_gpu_local_experts as experts
import test_gpu_local_linear as linear
from gpu_util import say, torch_cuda
from paper_1905_09598_amd import local

pytestmark = pytest.mark.gpu
T = linear.T


@pytest.fixture
def tiles(monkeypatch):
    """The tiles of the calls made: (forward's, backward's) as the library names them."""
    seen = {False: None, True: None}
    run = local._run

    def recording(name, call, backward, x):
        out = (C.c_int32 * 4)()
        assert getattr(local.lib(), f"som_{name}_route")(C.byref(call), backward, out) == 0
        seen[backward] = list(out)
        run(name, call, backward, x)

    monkeypatch.setattr(local, "_run", recording)
    return seen


# product, its tile (negative: operands through registers), n, inner, outer
LINEAR = {
    "fp32": [("y", 128, 10421, 212, 652), ("y", 256, 3795, 204, 3860), ("y", -128, 1425, 205, 4274),
             ("dx", 128, 2183, 3276, 204), ("dx", 256, 10139, 1428, 204),
             ("dx", -128, 4199, 1510, 205), ("dw", 128, 415, 1740, 4156),
             ("dw", 256, 429, 4820, 3228), ("dw", -128, 403, 4709, 1305)],
    "half": [("y", 128, 7601, 200, 520), ("y", 256, 2723, 200, 3016), ("y", -128, 9363, 202, 394),
             ("dx", 128, 11141, 328, 200), ("dx", 256, 3081, 2712, 200),
             ("dx", 256, 7313, 1098, 202), ("dx", -128, 3475, 1157, 203),
             ("dw", 128, 405, 2696, 1480), ("dw", 256, 407, 3739, 2266),
             ("dw", -128, 403, 2607, 1571)]}
LINEAR = [(dtype, *c) for dtype in T for c in LINEAR["fp32" if dtype == "fp32" else "half"]]


def _tile_of_linear(tiles, product):
    return {"y": tiles[False][0], "dx": tiles[True][0], "dw": tiles[True][1]}[product]


@pytest.mark.parametrize("dtype,product,tile,n,inner,outer", LINEAR)
def test_products(tiles, dtype, product, tile, n, inner, outer):
    torch_cuda()
    say("tiles", dtype, product, tile, n, inner, outer)
    x, w, b, r, dy = linear._case(n, inner, outer, T[dtype], seed=n)
    linear._check(x, w, b, r, dy, "gelu")
    assert _tile_of_linear(tiles, product) == tile


@pytest.mark.parametrize("dtype,product,tile,n,inner,outer",
                         [c for c in LINEAR if c[2] < 0])
def test_products_of_rows_with_nan_between(tiles, dtype, product, tile, n, inner, outer):
    # what follows a row is read with its last piece, and must not count
    say("gaps", dtype, product, tile, n, inner, outer)

    def strided(t):
        wide = torch.full((n, t.shape[1] + 6), float("nan"), dtype=t.dtype, device="cuda")
        v = wide[:, 3:3 + t.shape[1]]
        v.copy_(t)
        return v

    x, w, b, r, dy = linear._case(n, inner, outer, T[dtype], seed=n + 1)
    linear._check(strided(x), w, b, strided(r), strided(dy), "none")
    assert _tile_of_linear(tiles, product) == tile


# product, its tile, n, k, experts, inner, hidden, outer
EXPERTS = {
    "fp32": [("w1", 128, 5661, 3, 3, 212, 196, 180), ("w1", 256, 5032, 2, 3, 156, 804, 172),
             ("w1", -128, 6906, 2, 3, 237, 259, 169), ("w2", 128, 1882, 3, 2, 28, 156, 724),
             ("w2", 256, 6130, 2, 2, 36, 156, 668), ("w2", -128, 4655, 3, 5, 26, 159, 262),
             ("gate", 128, 5661, 3, 3, 212, 196, 180), ("gate", 256, 5032, 2, 3, 156, 804, 172),
             ("gate", -128, 6906, 2, 3, 237, 259, 169), ("dx", 128, 6791, 2, 2, 260, 164, 36),
             ("dx", 256, 4578, 3, 3, 580, 164, 36), ("dx", -128, 7341, 3, 5, 158, 161, 38),
             ("dw1", 128, 1227, 1, 4, 3420, 332, 36), ("dw1", 256, 341, 1, 4, 3604, 532, 28),
             ("dw1", -128, 1870, 1, 5, 3390, 213, 33), ("dw2", 128, 492, 2, 3, 68, 580, 2708),
             ("dw2", 256, 353, 1, 5, 60, 484, 3284), ("dw2", -128, 1391, 1, 4, 43, 258, 3574)],
    "half": [("w1", 128, 5991, 3, 2, 168, 200, 152), ("w1", 256, 3660, 3, 4, 152, 648, 184),
             ("w1", -128, 6142, 3, 4, 154, 214, 191), ("w2", 128, 5908, 1, 3, 40, 152, 648),
             ("w2", 256, 7541, 3, 2, 56, 152, 264), ("w2", -128, 1795, 3, 3, 78, 155, 715),
             ("gate", 128, 5991, 3, 2, 168, 200, 152), ("gate", 256, 3660, 3, 4, 152, 648, 184),
             ("gate", -128, 6142, 3, 4, 154, 214, 191), ("dx", 128, 4479, 3, 3, 264, 152, 24),
             ("dx", 256, 7354, 3, 2, 299, 150, 26), ("dx", -128, 2995, 2, 3, 662, 153, 39),
             ("dw1", 128, 621, 2, 4, 3368, 264, 104), ("dw1", 256, 414, 3, 4, 3400, 520, 40),
             ("dw1", -128, 912, 1, 3, 3241, 388, 196), ("dw2", 128, 820, 2, 5, 184, 200, 3288),
             ("dw2", 256, 1700, 1, 5, 56, 392, 3560), ("dw2", -128, 1709, 1, 5, 30, 194, 3462)]}
# one run of each size looks at all of its products
EXPERTS = {dtype: {c[2:]: [d[:2] for d in EXPERTS[how] if d[2:] == c[2:]] for c in EXPERTS[how]}
           for dtype, how in (("fp32", "fp32"), ("bf16", "half"), ("fp16", "half"))}
EXPERTS = [(dtype, *size, wanted) for dtype in EXPERTS for size, wanted in EXPERTS[dtype].items()]


@pytest.mark.parametrize("dtype,n,k,e,inner,hidden,outer,wanted", EXPERTS)
def test_experts(tiles, dtype, n, k, e, inner, hidden, outer, wanted):
    torch_cuda()
    say("tiles", dtype, n, k, e, inner, hidden, outer, wanted)
    x, r, w1, b1, w2, b2, res = experts._case(n, k, e, inner, hidden, outer, T[dtype], seed=n,
                                              popular=0.3)
    experts._check(x, r, w1, b1, w2, b2, res)
    names = dict(zip(("w1", "w2"), tiles[False]), **dict(zip(("gate", "dw2", "dx", "dw1"),
                                                             tiles[True])))
    assert all(names[product] == tile for product, tile in wanted), (names, wanted)


@pytest.mark.parametrize("dtype", T)
def test_local_linear_maps_in_large_tiles(tiles, dtype):
    # without w2: dy by slot, x by list, the products' rows in fp32
    sizes = ((3000, 3, 2, 3096, 520), (3000, 3, 2, 3097, 521))
    for n, k, e, inner, hidden in sizes:
        say("maps", dtype, n, k, e, inner, hidden)
        x, r, w1, b1, _, _, _ = experts._case(n, k, e, inner, hidden, hidden, T[dtype], seed=n,
                                              popular=0.3)
        experts._check(x, r, w1, b1, None, None, None)
        assert abs(tiles[True][0]) >= 128


def test_large_tiles_in_a_graph(tiles):
    # their LDS passes 64 KB, which a launch has to ask for
    half = torch.bfloat16
    for product, n, inner, outer in (("y", 2723, 200, 3016), ("dx", 3081, 2712, 200),
                                     ("dw", 407, 3739, 2266)):
        say("graph", product, n, inner, outer)
        x, w, b, r, dy = linear._case(n, inner, outer, half, seed=3)

        def step():
            y, z = local.linear(x, w, b, "gelu", r, keep=True)
            return (y, *local.linear_backward(dy, x, w, z, "gelu"))

        step()
        assert _tile_of_linear(tiles, product) == 256
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        for seed in range(3):
            x.copy_(linear._draw(40 + seed, n, inner, dtype=half))
            g.replay()
            torch.cuda.synchronize()
            for a, e in zip(out, step()):
                assert torch.equal(a, e)
            torch.cuda.synchronize()
