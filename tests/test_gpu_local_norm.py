"""Layer norm and its gradient against 64 bits: every element within a bound derived
from the roundings (layers_oracle)."""
import math

import pytest
import torch

import layers_oracle as O
import paper_1905_09598_amd as som
from gpu_util import say, torch_cuda
from paper_1905_09598_amd import local

pytestmark = pytest.mark.gpu
T = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _draw(seed, *shape, dtype, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g) + shift).to(dtype).cuda()


def _check(x, w, b, dy, beside, eps=1e-5):
    y, kept = local.norm(x, w, b, eps, keep=True)
    o = O.Norm(O.d(x), O.d(w), O.d(b), eps, x.dtype)
    O.close(y, o.y, "y")
    O.close(kept[:, :1], o.mean, "mean")
    O.close(kept[:, 1:], (o.rstd, o.rstd * o.rho), "rstd")
    assert torch.equal(local.norm(x, w, b, eps), y)
    got = local.norm_backward(dy, x, w, kept, beside)
    want = o.backward(O.d(dy), O.d(beside))
    O.close(got[0], want["dx"], "dx")
    if w is None:
        assert got[1] is None
    else:
        O.close(got[1], want["dweight"], "dweight")
    O.close(got[2], want["dbias"], "dbias")
    return y, kept, got


# rows of less than a piece, of a few lanes, of a wave, of a workgroup, at and past what
# a workgroup holds (16-bit rows of 16,384, fp32 of 16,384 and 12,288)
SIZES = [(1, 1), (3, 2), (5, 3), (70, 4), (9, 5), (40, 7), (3, 8), (200, 9), (17, 12), (33, 64),
         (5, 100), (300, 257), (64, 512), (7, 513), (20, 1000), (50, 1025), (3, 2048), (30, 2051),
         (11, 4545), (6, 8200), (5, 10000), (3, 12288), (2, 12289), (3, 16384), (3, 16392),
         (2, 20001), (1, 50003)]


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("n,width", SIZES)
def test_rows_of_every_length(n, width, dtype):
    torch_cuda()
    say("norm", n, width, dtype)
    t = T[dtype]
    _check(_draw(n, n, width, dtype=t, scale=1.5, shift=0.5),
           _draw(n + 1, width, dtype=t, scale=0.2, shift=1.0), _draw(n + 2, width, dtype=t),
           _draw(n + 3, n, width, dtype=t), _draw(n + 4, n, width, dtype=t))


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("n,width", [(4000, 24), (3001, 130), (2500, 700), (9000, 3), (70000, 16)])
def test_many_rows(n, width, dtype):
    t = T[dtype]
    _check(_draw(n, n, width, dtype=t), _draw(n + 1, width, dtype=t), _draw(n + 2, width, dtype=t),
           _draw(n + 3, n, width, dtype=t), None)


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("width", [6, 40, 600, 20000])
def test_absent_parts(width, dtype):
    t = T[dtype]
    x, dy = _draw(1, 9, width, dtype=t), _draw(2, 9, width, dtype=t)
    w, b = _draw(3, width, dtype=t), _draw(4, width, dtype=t)
    for ww, bb in ((None, None), (w, None), (None, b)):
        _check(x, ww, bb, dy, None)
    _, kept = local.norm(x, w, b, keep=True)
    assert local.norm_backward(dy, x, w, kept, bias=False)[2] is None
    dx, dw, db = local.norm_backward(dy, x, None, kept, bias=False)
    assert dw is None and db is None


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("width", [5, 61, 515, 16400])
@pytest.mark.parametrize("offset,gap", [(0, 8), (1, 3), (5, 0)])
def test_row_strides_and_odd_beginnings(width, offset, gap, dtype):
    t, n = T[dtype], 7

    def strided(seed):
        wide = torch.full((n, offset + width + gap), float("nan"), dtype=t, device="cuda")
        v = wide[:, offset:offset + width]
        v.copy_(_draw(seed, n, width, dtype=t))
        return v

    x, dy, beside = strided(1), strided(2), strided(3)
    w, b = _draw(4, width + 1, dtype=t)[1:], _draw(5, width + 3, dtype=t)[3:]
    y, kept, got = _check(x, w, b, dy, beside)
    y2, kept2 = local.norm(x.contiguous(), w.clone(), b.clone(), keep=True)
    assert torch.equal(y, y2) and torch.equal(kept, kept2)
    again = local.norm_backward(dy.contiguous(), x.contiguous(), w.clone(), kept, beside.contiguous())
    for u, v in zip(got, again):
        assert torch.equal(u, v)


@pytest.mark.parametrize("width", [12, 700, 4545])
def test_rows_far_from_zero(width):
    """Rows whose mean is 10,000 times their spread keep the bits that x has."""
    x = _draw(1, 20, width, dtype=torch.float32, shift=1e4)
    _check(x, None, None, _draw(2, 20, width, dtype=torch.float32), None)


@pytest.mark.parametrize("shift", [1.0, 1e4, 1e6])
@pytest.mark.parametrize("n,width", [(1, 3), (40, 7), (700, 40), (300, 257), (50, 1500), (9, 4545), (20, 12288),
                                     (5, 12289), (30, 20001)])
def test_gradients_of_rows_far_from_zero(n, width, shift):
    """As forward does, the gradients take the rounding of the mean that they read out of it."""
    x = _draw(1, n, width, dtype=torch.float32, shift=shift)
    x[::2] = -x[::2]
    w, dy = _draw(2, width, dtype=torch.float32, shift=1.0), _draw(3, n, width, dtype=torch.float32, shift=0.5)
    beside = _draw(4, n, width, dtype=torch.float32)
    _, kept = local.norm(x, w, keep=True)
    want = O.Norm(O.d(x), O.d(w), None, 1e-5, x.dtype).backward(O.d(dy), O.d(beside), found=True)
    for name, got in zip(("dx", "dweight", "dbias"), local.norm_backward(dy, x, w, kept, beside)):
        O.close(got, want[name], name)
    # each gradient by itself
    for wanted in ("dx", "dweight"):
        call = local._norm_call(x, w, 0.0)
        call.dy, call.lddy, call.kept = dy.data_ptr(), width, kept.data_ptr()
        call.beside, call.ldb = beside.data_ptr(), width
        out = torch.full_like(x if wanted == "dx" else w, 7.0)
        setattr(call, wanted, out.data_ptr())
        local._run("norm", call, True, x)
        O.close(out, want[wanted], wanted)


def test_constant_rows_and_other_ends():
    x = torch.full((4, 300), 3.25, device="cuda")
    y, kept = local.norm(x, eps=1e-5, keep=True)
    assert torch.equal(y, torch.zeros_like(y))
    assert torch.allclose(kept[:, 1], torch.full((4,), 1e-5 ** -0.5, device="cuda"), rtol=1e-6)
    dx, _, db = local.norm_backward(torch.ones_like(x), x, None, kept)
    assert float(dx.abs().max()) == 0 and torch.equal(db, torch.full_like(db, 4.0))
    x = _draw(2, 5, 300, dtype=torch.float32)
    x[1, 7], x[3, 0] = math.nan, math.inf
    y = local.norm(x)
    bad = torch.tensor([False, True, False, True, False], device="cuda")
    assert torch.equal(torch.isnan(y).all(1), bad) and torch.equal(torch.isnan(y).any(1), bad)


@pytest.mark.parametrize("width", [3, 40, 20000])
def test_no_rows(width):
    x = torch.empty(0, width, dtype=torch.bfloat16, device="cuda")
    w = _draw(1, width, dtype=torch.bfloat16)
    y, kept = local.norm(x, w, w, keep=True)
    assert y.shape == (0, width) and kept.shape == (0, 2)
    dx, dw, db = local.norm_backward(x, x, w, kept)
    assert dx.shape == (0, width)
    assert float(dw.abs().max()) == 0 and float(db.abs().max()) == 0


def test_offsets_beyond_32_bits():
    """Rows 2^31 elements and more behind the first."""
    wide = torch.empty((1 << 31) + 8192, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(wide, (3, 100), (1 << 30, 1))
    x.copy_(_draw(1, 3, 100, dtype=torch.bfloat16))
    y, kept = local.norm(x, keep=True)
    assert torch.equal(y, local.norm(x.contiguous()))
    dx, _, db = local.norm_backward(x, x, None, kept)
    again = local.norm_backward(x.contiguous(), x.contiguous(), None, kept)
    assert torch.equal(dx, again[0]) and torch.equal(db, again[2])


def test_streams_graphs_and_repeats():
    x, dy = _draw(1, 500, 1000, dtype=torch.bfloat16), _draw(2, 500, 1000, dtype=torch.bfloat16)
    w = _draw(3, 1000, dtype=torch.bfloat16)

    def once():
        y, kept = local.norm(x, w, w, keep=True)
        return (y, *local.norm_backward(dy, x, w, kept, y))

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
    x = _draw(1, 4, 16, dtype=torch.float32)
    w = x[0].clone()
    _, kept = local.norm(x, keep=True)
    bad = [
        (TypeError, lambda: local.norm(x.double())), (TypeError, lambda: local.norm(x.cpu())),
        (TypeError, lambda: local.norm(x, w.bfloat16())), (ValueError, lambda: local.norm(x, w[:8])),
        (ValueError, lambda: local.norm(x[0])), (ValueError, lambda: local.norm(x[:, :0])),
        (ValueError, lambda: local.norm(x.t())), (ValueError, lambda: local.norm(x, w.cpu().cuda()[::2])),
        (som.SomError, lambda: local.norm(x, eps=-1.0)),
        (som.SomError, lambda: local.norm(x, eps=math.nan)),
        (som.SomError, lambda: local.norm(x, eps=math.inf)),
        (TypeError, lambda: local.norm_backward(x, x, w, None)),
        (TypeError, lambda: local.norm_backward(x, x, w, kept.double())),
        (ValueError, lambda: local.norm_backward(x, x, w, kept[:3])),
        (ValueError, lambda: local.norm_backward(x[:3], x, w, kept)),
        (ValueError, lambda: local.norm_backward(x, x, w, kept, x[:, :8])),
        (ValueError, lambda: local.norm(x.clone().requires_grad_())),
    ]
    for error, call in bad:
        with pytest.raises(error):
            call()
