"""The optimizer step against 64 bits, and its 8-bit states against what their
format allows."""
import math

import pytest
import torch

import local_oracle as O
from gpu_util import say, torch_cuda
from paper_1905_09598_amd import local

pytestmark = pytest.mark.gpu
T = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HOW = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)


def _draw(seed, n, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(n, generator=g)).to(dtype).cuda()


def _pieces(flat, sizes):
    at, out = 0, []
    for n in sizes:
        out.append(flat[at:at + n])
        at += -(-n // 256) * 256
    return out


SIZES = [1, 255, 256, 257, 4, 5003, 2048, 0, 2049, 70001, 3]


def _held(opt, name, sizes):
    """A state's values as they stand for, in 64 bits, tensor by tensor."""
    t = O.d(getattr(opt, name).float())
    if opt.bits == 8:
        t = (t.view(-1, 256) * O.d(getattr(opt, name + "_scale")).unsqueeze(1)).view(-1)
        if name == "square":
            t = t * t
    return _pieces(t, sizes)


@pytest.mark.parametrize("master", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", T)
@pytest.mark.parametrize("dtype", T)
def test_steps(dtype, grad, bits, master):
    torch_cuda()
    say("adamw", dtype, grad, bits, master)
    dt = T[dtype]
    params = [_draw(i, n, dt) for i, n in enumerate(SIZES)]
    opt = local.AdamW(params, bits=bits, master=master, **HOW)
    b1, b2 = HOW["betas"]
    for step in (1, 2, 3):
        before = [O.d(p) for p in (_pieces(opt.master, SIZES) if master else params)]
        m0, v0 = _held(opt, "mean", SIZES), _held(opt, "square", SIZES)
        grads = [_draw(100 * step + i, n, T[grad], 1e-2) for i, n in enumerate(SIZES)]
        opt.step(grads)
        m1, v1 = _held(opt, "mean", SIZES), _held(opt, "square", SIZES)
        after = _pieces(opt.master, SIZES) if master else params
        for i, n in enumerate(SIZES):
            if not n:
                continue
            p, m, v = O.adamw(before[i], O.d(grads[i]), m0[i], v0[i], step, HOW["lr"], b1, b2,
                              HOW["eps"], HOW["weight_decay"])
            # 12 roundings of 32 bits on the way; m may cancel: its terms' magnitudes count
            size = b1 * m0[i].abs() + (1 - b1) * O.d(grads[i]).abs()
            move = HOW["lr"] * size / (1 - b1 ** step) / (
                (v / (1 - b2 ** step)).sqrt() + HOW["eps"])
            bound = 12 * O.V * (p.abs() + HOW["lr"] * p.abs() + move) + O.TINY[torch.float32]
            O.close(after[i], (p, bound + (0 if master else O.stored(p, dt))), "param")
            if master:
                O.close(params[i], (p, bound + O.stored(p, dt)), "param")
            if bits == 32:
                O.close(m1[i], (m, 4 * O.V * size + O.TINY[torch.float32]), "mean")
                O.close(v1[i], (v, 6 * O.V * v + O.TINY[torch.float32]), "square")
            else:
                for got, want, name in ((m1[i], m, "mean"), (v1[i].sqrt(), v.sqrt(), "root")):
                    for b in range(0, n, 256):
                        w = want[b:b + 256]
                        unit = w.abs().max() / 448
                        # e4m3: 2^-4 of a value, 2^-10 units below 2^-6 units (a root
                        # above 0 is never held as 0: then up to 2^-9)
                        low = 2.0 ** (-9 if name == "root" else -10)
                        bound = torch.maximum(w.abs() * 2.0 ** -4, unit * low) * (1 + 1e-5)
                        O.close(got[b:b + 256], (w, bound + 1e-36), name)
                        if name == "root":
                            assert ((got[b:b + 256] > 0) == (w > 0)).all()
    for name in ("mean", "square"):       # nothing is written between the tensors
        t = getattr(opt, name).float()
        used = torch.zeros_like(t, dtype=torch.bool)
        for piece in _pieces(used, SIZES):
            piece[:] = True
        assert not t[~used].any()


def test_odd_beginnings():
    # parameters and gradients that begin at any element of their storage
    store, gstore = _draw(1, 9000, torch.bfloat16), _draw(2, 9000, torch.bfloat16, 1e-2)
    views = [(1, 700), (703, 1025), (1730, 4001)]
    a = [store[o:o + n] for o, n in views]
    b = [t.clone() for t in a]
    oa, ob = local.AdamW(a, bits=8, **HOW), local.AdamW(b, bits=8, **HOW)
    rest = store.clone()
    for _ in range(3):
        oa.step([gstore[o:o + n] for o, n in views])
        ob.step([gstore[o:o + n].clone() for o, n in views])
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    keep = torch.ones(9000, dtype=torch.bool)
    for o, n in views:
        keep[o:o + n] = False
    assert torch.equal(store[keep], rest[keep])


def test_many_tensors_take_several_launches():
    params = [_draw(i, 300 + i) for i in range(600)]
    grads = [_draw(1000 + i, 300 + i) for i in range(600)]
    ref = [p.clone() for p in params]
    local.AdamW(params, **HOW).step(grads)
    for p, q, g in zip(params, ref, grads):
        local.AdamW([q], **HOW).step([g])
        assert torch.equal(p, q)


def test_resume_from_state():
    grads = [[_draw(10 * s + i, n, scale=1e-2) for i, n in enumerate((900, 77))] for s in range(4)]
    for bits in (32, 8):
        a = [_draw(1, 900), _draw(2, 77)]
        b = [t.clone() for t in a]
        whole = local.AdamW(a, bits=bits, **HOW)
        for g in grads:
            whole.step(g)
        first = local.AdamW(b, bits=bits, **HOW)
        first.step(grads[0]), first.step(grads[1])
        names = ["mean", "square"] + (["mean_scale", "square_scale"] if bits == 8 else [])
        state = {k: getattr(first, k).clone() for k in names}
        second = local.AdamW(b, bits=bits, step=2, state=state, **HOW)
        second.step(grads[2]), second.step(grads[3])
        assert all(torch.equal(x, y) for x, y in zip(a, b))
        first.close()
        first.close()


def test_zero_huge_and_spoilt_gradients():
    for bits in (32, 8):
        p = [_draw(1, 1024)]
        start = p[0].clone()
        opt = local.AdamW(p, lr=0.1, weight_decay=0.0, bits=bits)
        opt.step([torch.zeros(1024, device="cuda")])
        assert torch.equal(p[0], start)             # 0 / eps
        g = torch.zeros(1024, device="cuda")
        g[3], g[300] = 1e18, 1e-20                   # far apart in one block, tiny in another
        opt.step([g])
        assert torch.isfinite(p[0]).all()
        opt.step([torch.zeros(1024, device="cuda")])
        assert torch.isfinite(p[0]).all()
        assert float((p[0] - start).abs().max()) < 1.0
        g[700] = math.nan
        opt.step([g])
        bad = torch.isnan(p[0])
        assert bad[700] and int(bad.sum()) == 1
        opt.step([torch.zeros(1024, device="cuda")])  # 8 bits: its block shares the scale
        assert not torch.isnan(p[0][:512]).any() and torch.isnan(p[0][700])


def test_capture_into_a_graph():
    p, q = [_draw(1, 5000, torch.bfloat16)], [_draw(1, 5000, torch.bfloat16)]
    g = [_draw(2, 5000, torch.bfloat16)]
    a, b = local.AdamW(p, bits=8, **HOW), local.AdamW(q, bits=8, **HOW)
    graph = torch.cuda.CUDAGraph()
    a.steps = b.steps = 4
    with torch.cuda.graph(graph):
        a.step(g)
    for s in range(3):
        g[0].copy_(_draw(3 + s, 5000, torch.bfloat16))
        b.steps = 4                # the captured step's number is part of the graph
        graph.replay()
        torch.cuda.synchronize()
        b.step(g)
        assert torch.equal(p[0], q[0]) and torch.equal(a.mean.view(torch.uint8),
                                                       b.mean.view(torch.uint8))


def test_refusals():
    p = [_draw(1, 100)]
    for bad in (dict(bits=16), dict(state={"mean": p[0], "square": p[0]})):
        with pytest.raises(ValueError):
            local.AdamW(p, **bad)
    with pytest.raises(ValueError):
        local.AdamW([])
    with pytest.raises(TypeError):
        local.AdamW([p[0].double()])
    with pytest.raises(ValueError):
        local.AdamW([p[0].view(10, 10).t()])
    opt = local.AdamW(p)
    with pytest.raises(ValueError):
        opt.step([])
    with pytest.raises(ValueError):
        opt.step([p[0][:99]])
    with pytest.raises(TypeError):
        opt.step([p[0].cpu()])
    opt.betas = (1.0, 0.9)
    with pytest.raises(local.SomError):
        opt.step([p[0].clone()])
    opt.betas, opt.lr = (0.9, 0.9), math.inf
    with pytest.raises(local.SomError):
        opt.step([p[0].clone()])
