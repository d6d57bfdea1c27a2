"""The operators run together: a map, the gate made from it, routing, experts and
the optimizer."""
import importlib.util
import os

import pytest
import torch

import paper_1905_09598_amd as som
from gpu_util import say, torch_cuda
from paper_1905_09598_amd import local

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location(
        "local_models", os.path.join(ROOT, "examples", "local_models.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_example_learns_what_one_linear_model_cannot():
    torch_cuda()
    got = _example().run(n=4000, steps=200, say=say)
    assert got["last"] < 0.2 * got["first"]
    assert got["last"] < got["linear"]
    assert got["same"] > 0.9           # bf16 prototypes against fp32 distances
    assert got["alone"] < 0.05


def test_gate_from_map_chooses_the_best_matching_units():
    # fp32: the order of the scores is that of the distances, but for near ties
    g = torch.Generator().manual_seed(0)
    x = torch.randn(500, 40, generator=g).cuda()
    m = som.Map(5, 7, 40, seed=3)
    m.weights = torch.randn(35, 40, generator=g)
    bmu, second, d1 = m.bmu(x, second=True)
    w, b = local.gate_from_map(m.weights, tau=3.0)
    r = local.route(local.linear(x, w, b), k=2)
    d = torch.cdist(x.double(), m.weights.double()).square().sort(1).values
    clear = ((d[:, 1] - d[:, 0] > 1e-4 * d[:, 0]) & (d[:, 2] - d[:, 1] > 1e-4 * d[:, 1]))
    assert int(clear.sum()) > 450
    assert torch.equal(r.index[clear, 0], bmu[clear]) and torch.equal(r.index[clear, 1],
                                                                      second[clear])
    # the weights are the softmax of -d / (2 tau) over the two
    want = torch.softmax(-d[:, :2] / 6.0, 1)
    assert float((r.weight.double()[clear] - want[clear]).abs().max()) < 1e-4
    # hard routing by the map itself
    hard = local.dispatch(torch.stack([bmu, second], 1).contiguous(), None, 35)
    assert int(hard.offsets[-1]) == 1000
    with pytest.raises(ValueError):
        local.gate_from_map(m.weights, tau=0.0)
