"""The README's calls as they are written, on a small map and few documents."""
import os
import re

import pytest
import torch

import layers_oracle as O
from gpu_util import torch_cuda

pytestmark = pytest.mark.gpu
README = os.path.join(os.path.dirname(os.path.dirname(__file__)), "README.md")


def _blocks():
    """Its Python blocks, in order, with smaller sizes."""
    found = re.findall(r"```python\n(.*?)```", open(README).read(), re.S)
    assert len(found) == 3
    for a, b in (("rand(100000, 2048", "rand(600, 64"), ("Map(100, 100, 2048", "Map(10, 10, 64"),
                 ("epochs=5", "epochs=2"), ("sigma0=50.0", "sigma0=5.0")):
        assert a in found[0]
        found[0] = found[0].replace(a, b)
    return found


def test_the_calls_in_order():
    torch_cuda()
    torch.manual_seed(3)
    n, d, units, hidden = 600, 64, 100, 40
    train, experts, student = _blocks()
    names = {}
    exec(train, names)
    assert names["bmu"].shape == (n,) and names["W"].shape == (units, d)

    def draw(*shape, scale=1.0):
        return scale * torch.randn(*shape, device="cuda")

    names.update(w1=draw(units, hidden, d, scale=d ** -0.5), b1=draw(units, hidden, scale=0.1),
                 w2=draw(units, d, hidden, scale=hidden ** -0.5), b2=draw(units, d, scale=0.1), dy=draw(n, d))
    exec(experts, names)
    assert names["y"].shape == (n, d) and names["dw"].shape == (units, d)
    for t in (names["g"].x, names["g"].w1, names["dx"], names["dw"], names["db"]):
        assert torch.isfinite(t).all()

    half = torch.bfloat16                       # as a head in 8 bits takes it
    made = dict(X=names["X"], nw=1 + draw(d, scale=0.1), nb=draw(d, scale=0.1),
                w1=draw(2, hidden, d, scale=d ** -0.5), b1=draw(2, hidden, scale=0.1),
                w2=draw(d, hidden, scale=hidden ** -0.5), b2=draw(d, scale=0.1),
                wh=draw(units, d, scale=d ** -0.5), bh=draw(units, scale=0.1))
    names.update({k: t.to(half) for k, t in made.items()})
    names["labels"] = torch.randint(-1, units, (n,), device="cuda", dtype=torch.int32)
    exec(student, names)
    scores, index = names["scores"], names["r"].index
    # the rest keeps its bits: every term is positive, off by a softmax's and a sum's roundings
    p = scores.double().softmax(1).scatter(1, index.long(), 0.0).sum(1)
    size = (scores - scores.max(1, keepdim=True).values).abs().max(1).values.double()
    assert ((names["rest"].double() - p).abs() <= (units + 4 * size + 40) * O.V * p).all()
    assert names["loss"].shape == (n,) and torch.isfinite(names["loss"]).all()
    for k, of in (("dx", "X"), ("dnw", "nw"), ("dw1", "w1"), ("db1", "b1"), ("dw2", "w2"), ("dwh", "wh"), ("dbh", "bh")):
        assert names[k].shape == names[of].shape and torch.isfinite(names[k]).all(), k
    assert names["s"].shape == (n, units) and torch.isfinite(names["s"]).all()
