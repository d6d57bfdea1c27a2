"""Distillation and its gradient against 64 bits: every element within a bound derived
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


def _inputs(n, classes, k, dtype, seed=0, teacher=torch.float32):
    g = torch.Generator().manual_seed(seed)
    s = (2.5 * torch.randn(n, classes, generator=g)).to(dtype).cuda()
    index = torch.stack([torch.randperm(max(classes, k), generator=g)[:k] for _ in range(min(n, 50))])
    index = index.repeat(-(-n // 50), 1)[:n].int().cuda()      # beyond the classes: absent
    t = (2 * torch.randn(n, k, generator=g)).to(teacher).cuda()
    rest = (0.6 * torch.rand(n, generator=g)).cuda()
    label = torch.randint(-1, classes + 1, (n,), generator=g).int().cuda()
    dloss = (0.1 + torch.rand(n, generator=g)).cuda()
    return s, index, t, rest, label, dloss


def _check(s, index, t, heat, rest, label, mix, dloss):
    loss, dlogits = local.distill(s, index, t, heat, rest, label, mix, dloss)
    o = O.Distill(O.d(s), index, O.d(t), heat, O.d(rest), label, mix, O.d(dloss), s.dtype)
    O.close(loss, o.loss, "loss")
    O.close(dlogits, o.dlogits, "dlogits")
    assert torch.equal(local.distill(s, index, t, heat, rest, label, mix).nan_to_num(), loss.nan_to_num())
    back = local.distill_backward(dloss, s, index, t, heat, rest, label, mix)
    assert torch.equal(back.nan_to_num(), dlogits.nan_to_num())
    return loss, dlogits


# rows of less than a piece, of a few lanes, of a wave, of a workgroup, at and past what
# a workgroup holds (16-bit rows of 32,768 and 65,536, fp32 of 16,384 and 32,768)
SIZES = [(1, 1, 1), (5, 2, 1), (70, 3, 2), (9, 7, 3), (200, 8, 2), (17, 9, 4), (33, 64, 8),
         (100, 100, 4), (7, 257, 64), (20, 513, 3), (3, 1024, 5), (40, 1025, 8), (6, 4545, 16),
         (3, 10000, 8), (2, 16385, 4), (2, 32768, 9), (2, 32769, 7), (2, 50001, 8), (2, 65536, 8),
         (2, 65545, 30), (1, 200003, 32)]


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("n,classes,k", SIZES)
def test_rows_of_every_length(n, classes, k, dtype):
    torch_cuda()
    say("distill", n, classes, k, dtype)
    s, index, t, rest, label, dloss = _inputs(n, classes, k, T[dtype], seed=n + classes)
    _check(s, index, t, 2.0, rest, label, 0.6, dloss)
    _check(s, index, t, 1.0, None, None, 1.0, dloss)


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("classes", [6, 300, 2051])
def test_parts_and_temperatures(classes, dtype):
    s, index, t, rest, label, dloss = _inputs(60, classes, 5, T[dtype], seed=7, teacher=T[dtype])
    for heat in (0.25, 1.5, 10.0):
        for r in (None, rest):
            _check(s, index, t, heat, r, label, 0.3, dloss)
            _check(s, index, t, heat, r, None, 1.0, dloss)
            _check(s, index, t, heat, r, label, 1.0, dloss)     # labels of no weight
        _check(s, index, t, heat, rest, label, 0.0, dloss)      # a teacher of no weight
    loss, dlogits = local.distill(s, label=label, mix=0.0, dloss=0.5)
    o = O.Distill(O.d(s), None, None, 1.0, None, label, 0.0, torch.full_like(O.d(dloss), 0.5), s.dtype)
    O.close(loss, o.loss, "loss")
    O.close(dlogits, o.dlogits, "dlogits")


@pytest.mark.parametrize("classes", [5, 130, 5000, 70001])
def test_absent_repeated_and_closed_classes(classes):
    s, index, t, rest, label, dloss = _inputs(40, classes, 6, torch.float32, seed=11)
    label = label.clamp(0, classes - 1)
    index[0], index[1, :3], index[2, 1:] = -1, -5, classes + 7
    index[3] = index[3, 0]                       # one class, six times
    index[4, 1], index[5, 2:4] = index[4, 0], index[5, 0]
    t[6], t[7, 2] = -math.inf, -math.inf
    s[8:16][torch.rand(8, classes, generator=torch.Generator().manual_seed(1)).cuda() < 0.5] = -math.inf
    s[8:16, 0] = 1.0
    s[16] = -math.inf                            # a row without an open class
    s[17], s[18] = torch.finfo(torch.float32).min, -1e38
    s[18, classes // 2] = 3e38
    rest[19], rest[20], rest[21], rest[22] = 0.0, 1.0, -1e-7, 1.5
    loss, dlogits = _check(s, index, t, 2.0, rest, label, 0.5, dloss)
    assert float(loss[16]) == 0 and float(dlogits[16].abs().max()) == 0
    loss, dlogits = _check(s, index, t, 1.0, None, None, 1.0, dloss)
    assert float(loss[0]) == 0 and float(dlogits[0].abs().max()) == 0
    assert float(loss[6]) == 0 and float(dlogits[6].abs().max()) == 0


@pytest.mark.parametrize("classes", [6, 700, 80000])
def test_the_rest_without_another_class(classes):
    """All open classes are named: what is left for the others is lost (infinity)."""
    s, _, t, rest, _, dloss = _inputs(4, classes, 3, torch.float32, seed=3)
    index = torch.tensor([[0, 1, 2]] * 4, dtype=torch.int32, device="cuda")
    s[:, 3:] = -math.inf
    rest[1] = 0.0
    loss, dlogits = _check(s, index, t, 1.0, rest, None, 1.0, dloss)
    assert torch.isinf(loss).tolist() == [True, False, True, True]
    assert torch.isfinite(dlogits).all() and float(dlogits[:, 3:].abs().max()) == 0


@pytest.mark.parametrize("classes", [6, 700, 80000])
def test_numbers_that_are_none(classes):
    s, index, t, rest, label, dloss = _inputs(8, classes, 3, torch.float32, seed=4)
    index = index.clamp(0, classes - 1)
    s[1, classes - 1], s[2, 0], t[3, 1], t[4, 0] = math.nan, math.inf, math.nan, math.inf
    s[5, 2], s[5, 3:] = math.nan, -math.inf
    s[5, :2] = -math.inf
    loss, dlogits = local.distill(s, index, t, 1.0, rest, label.clamp(0, classes - 1), 0.5, dloss)
    bad = torch.tensor([False, True, True, True, True, True, False, False], device="cuda")
    assert torch.equal(torch.isnan(loss), bad)
    assert torch.equal(torch.isnan(dlogits).all(1), bad) and torch.equal(torch.isnan(dlogits).any(1), bad)


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("classes", [6, 23, 300, 1030, 9000, 66000])
def test_named_classes_far_ahead_of_the_others(classes, dtype):
    """What the teacher leaves out is far below what it names, further than an exponential
    reaches: loss and gradient are numbers like others, in rows of a lane, a wave, a
    workgroup and beyond one."""
    say("far ahead", classes, dtype)
    heat = 2.0 if dtype == "fp32" else 0.5
    s, _, t, rest, label, dloss = _inputs(24, classes, 3, T[dtype], seed=21)
    index = torch.randint(0, classes, (24, 3), generator=torch.Generator().manual_seed(1)).int().cuda()
    rest, label = rest + 0.2, label.clamp(0, classes - 1)
    gaps = torch.tensor([30, 40, 43, 60, 80, 86, 87, 88, 90, 95, 103, 110, 130, 160, 200, 400], device="cuda")
    named = torch.zeros(24, classes, dtype=torch.bool, device="cuda").scatter_(1, index.long(), True)
    s[:16] = torch.where(named[:16], s[:16], (s[:16] - heat * gaps[:, None]).to(s.dtype))
    s[3:16:4][named[3:16:4]] = 1.0                       # equal leaders
    others = ~named[4:8] & (torch.rand(4, classes, generator=torch.Generator().manual_seed(2)) < 0.5).cuda()
    s[4:8] = s[4:8].masked_fill(others, -math.inf)       # closed classes among them
    s[16:20] = s[16:20].masked_fill(named[16:20], -math.inf)      # and none of the named open
    s[20:22] = torch.where(named[20:22], s[20:22] - 300, s[20:22])
    s[22:24] = torch.where(named[22:24], s[22:24], (s[22:24] * 2.0 - 500).to(s.dtype))
    loss, dlogits = _check(s, index, t, heat, rest, None, 1.0, dloss)
    assert torch.isfinite(loss[:4]).all() and torch.isfinite(loss[8:16]).all()
    some = ~named[:16] & (s[:16] > -math.inf)
    assert float(dlogits[:16][some].max()) <= 0 and float(dlogits[:16][some].min()) < -1e-3 / classes
    _check(s, index, t, heat, rest, label, 0.5, dloss)
    _check(s, index, t, 1.0, rest, label, 0.5, dloss)
    if dtype == "fp32":
        _check(s, index, t, 2.0 ** -20, rest, label, 0.5, dloss)


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("classes", [6, 30, 700, 12000, 80000])
def test_numbers_that_are_none_in_rows_without_parts(classes, dtype):
    """Neither a teacher's class nor a label: 0 and 0, unless a logit is none."""
    s, index, t, rest, label, dloss = _inputs(12, classes, 3, T[dtype], seed=4)
    index[:8], label[:10] = -1, -1
    s[1, classes - 1], s[2, 0], s[3, 1], s[8, 2] = math.nan, math.inf, math.nan, math.inf
    s[3, 2:] = -math.inf
    t[4, 1], t[5] = math.nan, math.inf             # of classes that are not there
    bad = torch.tensor([i in (1, 2, 3, 8) for i in range(12)], device="cuda")
    for said, mix in (((index, t, 1.0, rest, label), 0.5), ((index, t, 2.0, rest, None), 1.0),
                      ((index, t, 1.5, None, label), 0.5), ((None, None, 1.0, None, label), 0.0)):
        loss, dlogits = local.distill(s, *said, mix, dloss)
        assert torch.equal(torch.isnan(loss), bad)
        assert torch.equal(torch.isnan(dlogits).all(1), bad) and torch.equal(torch.isnan(dlogits).any(1), bad)
        still = torch.tensor([0, 4, 5, 6, 7], device="cuda")
        assert float(loss[still].abs().max()) == 0 and float(dlogits[still].abs().max()) == 0


def test_a_teacher_that_the_student_matches():
    """Every class named, the same logits: loss and gradient are 0 to rounding."""
    s = torch.randn(10, 50, generator=torch.Generator().manual_seed(1)).cuda()
    index = torch.arange(50, dtype=torch.int32, device="cuda").expand(10, 50).contiguous()
    loss, dlogits = local.distill(s, index, s.clone(), 3.0, dloss=1.0)
    assert float(loss.abs().max()) < 9 * 50 * 2 ** -20 and float(dlogits.abs().max()) < 3 * 2 ** -18


@pytest.mark.parametrize("classes", [7, 301, 4001, 66000])
@pytest.mark.parametrize("offset,gap", [(0, 8), (1, 3), (5, 0)])
def test_row_strides_and_odd_beginnings(classes, offset, gap):
    s, index, t, rest, label, dloss = _inputs(6, classes, 4, torch.bfloat16, seed=2)
    wide = torch.full((6, offset + classes + gap), float("nan"), dtype=s.dtype, device="cuda")
    v = wide[:, offset:offset + classes]
    v.copy_(s)
    for u, w in zip(local.distill(v, index, t, 2.0, rest, label, 0.5, dloss),
                    local.distill(s, index, t, 2.0, rest, label, 0.5, dloss)):
        assert torch.equal(u, w)


def test_rows_beyond_the_last_are_left_and_none_are_fine():
    s, index, t, rest, label, dloss = _inputs(3, 40, 2, torch.float32, seed=5)
    held = torch.full((8, 40), 7.0, device="cuda")
    call = local._distill_call(s, index, t, 1.0, rest, label, 0.5, dloss)
    loss = torch.full((8,), 7.0, device="cuda")
    call.loss, call.dlogits = loss.data_ptr(), held.data_ptr()
    som._check(local.lib().som_distill(local.C.byref(call)), "som_distill")
    assert torch.equal(held[3:], torch.full_like(held[3:], 7.0)) and float(loss[3:].min()) == 7
    loss, dlogits = local.distill(s[:0], index[:0], t[:0], 1.0, rest[:0], label[:0], 0.5, dloss[:0])
    assert loss.shape == (0,) and dlogits.shape == (0, 40)


@pytest.mark.parametrize("classes", [7, 300, 5000, 70000])
def test_gradient_in_the_logits_place(classes):
    s, index, t, rest, label, dloss = _inputs(9, classes, 4, torch.bfloat16, seed=2)
    want = local.distill(s, index, t, 2.0, rest, label, 0.5, dloss)
    call = local._distill_call(s, index, t, 2.0, rest, label, 0.5, dloss)
    loss = torch.empty(9, device="cuda")
    call.loss, call.dlogits = loss.data_ptr(), s.data_ptr()
    som._check(local.lib().som_distill(local.C.byref(call)), "som_distill")
    assert torch.equal(loss, want[0]) and torch.equal(s, want[1])


def test_gradient_over_other_rows_logits_is_refused():
    s, index, t, rest, label, dloss = _inputs(4, 40, 2, torch.float32, seed=5)
    room = torch.zeros(4 * 48 + 200, device="cuda")
    at = room.data_ptr()
    loss = torch.empty(4, device="cuda")

    def run(n, lds, first, to):
        call = local._distill_call(s, index, t, 1.0, rest, label, 0.5, dloss)
        call.n, call.lds, call.logits, call.dlogits, call.loss = n, lds, at + 4 * first, at + 4 * to, loss.data_ptr()
        return som.STATUS[local.lib().som_distill(local.C.byref(call))]

    for n, lds, first, to in ((4, 48, 0, 0), (2, 41, 8, 8), (4, 40, 0, 4), (4, 40, 4, 0), (3, 48, 0, 135),
                              (3, 48, 119, 0), (1, 40, 0, 39)):
        assert run(n, lds, first, to) == "SOM_E_ARG", (n, lds, first, to)
    for n, lds, first, to in ((4, 40, 0, 0), (1, 48, 0, 0), (3, 48, 0, 136), (3, 48, 120, 0)):
        assert run(n, lds, first, to) == "SOM_OK", (n, lds, first, to)


@pytest.mark.parametrize("heat", [2.0 ** -20, 2.0 ** 20])
def test_temperatures_at_their_ends(heat):
    s, index, t, rest, label, dloss = _inputs(30, 90, 4, torch.float32, seed=8)
    _check(s, index, t, heat, rest, label, 0.5, dloss)


@pytest.mark.parametrize("classes", [6, 700, 40000])
def test_low_temperatures_of_far_logits(classes):
    """Distances that pass fp32's range over the temperature, and losses that do not."""
    s, _, t, rest, label, dloss = _inputs(6, classes, 3, torch.float32, seed=23)
    index = torch.tensor([[1, 2, 3]] * 6, dtype=torch.int32, device="cuda")
    s[0, 1], s[1, 0], s[2, 4:], s[3, 1:4] = -3e37, 2e38, -1e38, -2e38
    s[4], s[4, 2], s[5, 1], s[5, 0] = -1e30, 1e38, -3e38, 3e38
    for heat in (2.0 ** -20, 2.0 ** -4, 0.125):
        loss, _ = _check(s, index, t, heat, rest, None, 1.0, dloss)
        assert torch.isfinite(loss).all()
        _check(s, index, t, heat, rest, label, 0.5, dloss)


@pytest.mark.parametrize("classes", [6, 700, 40000])
def test_low_temperatures_of_a_far_teacher(classes):
    """A teacher's logits that pass fp32's range over the temperature: they count by their
    differences."""
    s, _, t, rest, _, dloss = _inputs(6, classes, 3, torch.float32, seed=24)
    index = torch.tensor([[1, 2, 3]] * 6, dtype=torch.int32, device="cuda")
    t[0], t[1], t[2, 0], t[3, 1], t[4, 2] = 1e38, -3e38, 2e38, -1e38, -math.inf
    t[5, 0], t[5, 1] = 3e38, -3e38
    for heat in (2.0 ** -20, 2.0 ** -4, 0.5):
        loss, _ = _check(s, index, t, heat, rest, None, 1.0, dloss)
        assert torch.isfinite(loss).all() and float(loss.min()) > 0


def test_many_rows_and_offsets_beyond_32_bits():
    for n, classes, k in ((100001, 12, 3), (30001, 70, 40), (9000, 400, 8), (6001, 1003, 5),
                          (5003, 1900, 4)):
        s, index, t, rest, label, dloss = _inputs(n, classes, k, torch.bfloat16, seed=9)
        _check(s, index, t, 1.0, rest, label, 0.5, dloss)
    wide = torch.empty((1 << 31) + 4096, dtype=torch.bfloat16, device="cuda")
    v = torch.as_strided(wide, (3, 900), (1 << 30, 1))
    s, index, t, rest, label, dloss = _inputs(3, 900, 3, torch.bfloat16, seed=9)
    v.copy_(s)
    for u, w in zip(local.distill(v, index, t, 2.0, rest, label, 0.5, dloss),
                    local.distill(s, index, t, 2.0, rest, label, 0.5, dloss)):
        assert torch.equal(u, w)


@pytest.mark.parametrize("dtype", T)
@pytest.mark.parametrize("n,classes,k", [(100001, 12, 3), (30001, 70, 40), (9000, 230, 8), (9000, 400, 8),
                                         (6001, 1003, 5), (5003, 520, 4)])
def test_many_rows_of_few_lanes(n, classes, k, dtype):
    """Of many short rows a lane takes up to four pieces; rows whose named classes lead far
    beside rows in the same wave where they do not."""
    say("many rows", n, classes, k, dtype)
    s, index, t, rest, label, dloss = _inputs(n, classes, k, T[dtype], seed=classes)
    named = torch.zeros(n, classes + 1, dtype=torch.bool, device="cuda")
    named.scatter_(1, torch.where((index >= 0) & (index < classes), index, classes).long(), True)
    far = torch.arange(n, device="cuda")[:, None] % 7 == 3
    s = torch.where(far & ~named[:, :classes], s - 120, s)
    _check(s, index, t, 1.0, rest, label, 0.5, dloss)
    _check(s, index, t, 1.5, rest, None, 1.0, dloss)
    # the same document in a small batch, where a row is on more lanes: within their roundings
    part = torch.cat([torch.arange(40), torch.arange(n - 9, n)]).cuda()
    _check(s[part], index[part], t[part], 1.5, rest[part], None, 1.0, dloss[part])


@pytest.mark.parametrize("classes", [3000, 75233])
@pytest.mark.parametrize("share", [0.01, 0.99])
def test_shares_next_to_one(classes, share):
    """What the teacher names, or what it does not, is a hundredth, and the student agrees
    to a tenth of that: a loss of about 1e-4 made of terms of about 10.  The shares come
    from the smaller part of the sum: off by at most (classes + 40) V of themselves, and
    the loss with them; each named class's logarithms, of magnitudes up to 20 in all, by
    8 V of that, times the named share."""
    g = torch.Generator().manual_seed(13)
    n, k = 40, 8
    s = torch.randn(n, classes, generator=g, dtype=torch.float64)
    index = torch.stack([torch.randperm(classes, generator=g)[:k] for _ in range(n)])
    s.scatter_(1, index, -100.0)
    others = s.exp().sum(1)
    named = (others * share / (1 - share) / k).log().unsqueeze(1)
    s.scatter_(1, index, (named + 0.1 * torch.randn(n, k, generator=g)).double())
    s = s.float().cuda()
    index, t = index.int().cuda(), (0.1 * torch.randn(n, k, generator=g)).cuda()
    rest = torch.full((n,), 1 - share, device="cuda")
    ones = torch.ones(n, device="cuda")
    loss, dlogits = local.distill(s, index, t, 1.0, rest, dloss=1.0)
    o = O.Distill(O.d(s), index, O.d(t), 1.0, O.d(rest), None, 1.0, O.d(ones), torch.float32)
    V = O.V
    least = min(share, 1 - share)
    allowed = share * 8 * V * 20 + 8 * V * least + 4 * V * o.loss[0].abs()
    # a sum of positive terms in parts of at most 200 and their joins, not one chain
    allowed = allowed + least * (200 + 40) * V * 2
    assert ((loss.double() - o.loss[0]).abs() < allowed).all(), float(
        ((loss.double() - o.loss[0]).abs() / allowed).max())
    O.close(dlogits, o.dlogits, "dlogits")


def test_from_a_routing():
    """A map's nearest units teach a gate: the routing's index, its scores and its rest."""
    g = torch.Generator().manual_seed(6)
    scores, s = (torch.randn(200, 64, generator=g).cuda() for _ in range(2))
    r = local.route(scores, 4, renormalise=False)
    t = scores.gather(1, r.index.long())
    rest = (1 - r.weight.sum(1)).clamp(min=0)
    loss, dlogits = _check(s, r.index, t, 1.0, rest, None, 1.0, torch.ones(200, device="cuda"))
    # at the same scores the gate is right
    loss, dlogits = local.distill(scores, r.index, t, 1.0, rest, dloss=1.0)
    assert float(dlogits.abs().max()) < 2 ** -20 and float(loss.abs().max()) < 2 ** -18


def test_streams_graphs_and_repeats():
    s, index, t, rest, label, dloss = _inputs(300, 3000, 8, torch.bfloat16, seed=1)

    def once():
        return local.distill(s, index, t, 2.0, rest, label, 0.5, dloss)

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
        s.copy_(_inputs(300, 3000, 8, torch.bfloat16, seed=seed)[0])
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(held, once()):
            assert torch.equal(u, v)


def test_refusals():
    s, index, t, rest, label, dloss = _inputs(4, 16, 2, torch.float32)
    bad = [
        (TypeError, lambda: local.distill(s.double(), index, t)),
        (TypeError, lambda: local.distill(s.cpu(), index, t)),
        (ValueError, lambda: local.distill(s[0], index, t)),
        (ValueError, lambda: local.distill(s[:, :0], index, t)),
        (ValueError, lambda: local.distill(s, index)), (ValueError, lambda: local.distill(s, None, t)),
        (TypeError, lambda: local.distill(s, index.long(), t)),
        (ValueError, lambda: local.distill(s, index[:3], t)),
        (ValueError, lambda: local.distill(s, index[:, :0], t[:, :0])),
        (ValueError, lambda: local.distill(s, index, t[:, :1])),
        (TypeError, lambda: local.distill(s, index, t.double())),
        (TypeError, lambda: local.distill(s, index, t, rest=rest.double())),
        (ValueError, lambda: local.distill(s, index, t, rest=rest[:2])),
        (TypeError, lambda: local.distill(s, index, t, label=label.long(), mix=0.5)),
        (TypeError, lambda: local.distill(s, index, t, dloss=dloss.double())),
        (ValueError, lambda: local.distill(s, index, t, dloss=dloss[:1])),
        (ValueError, lambda: local.distill(s.clone().requires_grad_(), index, t)),
        (som.SomError, lambda: local.distill(s, index, t, temperature=0.0)),
        (som.SomError, lambda: local.distill(s, index, t, temperature=-1.0)),
        (som.SomError, lambda: local.distill(s, index, t, temperature=2.0 ** -21)),
        (som.SomError, lambda: local.distill(s, index, t, temperature=math.inf)),
        (som.SomError, lambda: local.distill(s, index, t, temperature=math.nan)),
        (som.SomError, lambda: local.distill(s, index, t, label=label, mix=1.5)),
        (som.SomError, lambda: local.distill(s, index, t, mix=0.5)),
        (som.SomError, lambda: local.distill(s, label=label, mix=0.5)),
        (som.SomError, lambda: local.distill(s, index, t, dloss=math.inf)),
        (som.SomError, lambda: local.distill(s.new_zeros(4, 200), torch.zeros(
            4, 65, dtype=torch.int32, device="cuda"), torch.zeros(4, 65, device="cuda"))),
    ]
    for error, call in bad:
        with pytest.raises(error):
            call()
