"""The local models' operators at the ends of their types' ranges, and calls that
have to be refused there."""
import math

import pytest
import torch

import local_oracle as O
from gpu_util import say, torch_cuda
from paper_1905_09598_amd import local

pytestmark = pytest.mark.gpu


def _draw(seed, *shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(dtype).cuda()


@pytest.mark.parametrize("n", [3, 200])
def test_relu_passes_the_gradient_of_a_z_that_rounds_to_zero(n):
    # z = 2^-26 is positive, and 0 in fp16; -2^-26 is not positive
    torch_cuda()
    say("relu next to 0", n)
    half = torch.float16
    x, w = torch.zeros(n, 16, dtype=half, device="cuda"), torch.zeros(8, 16, dtype=half,
                                                                      device="cuda")
    x[:, 0], w[:4, 0], w[4:, 0] = 2.0 ** -12, 2.0 ** -14, -2.0 ** -14
    w[:, 1] = 1.0                       # what dx shows
    y, z = local.linear(x, w, None, "relu", keep=True)
    dx, dw, db = local.linear_backward(torch.ones_like(y), x, w, z, "relu")
    assert (dx[:, 1] == 4).all()
    assert db.tolist() == [n] * 4 + [0] * 4
    assert (dw[:4, 0] > 0).all() and not dw[4:].any()
    # the experts' first layer
    index = torch.zeros(n, 1, dtype=torch.int32, device="cuda")
    r = local.dispatch(index, None, 1)
    w1, w2 = w.unsqueeze(0).contiguous(), torch.ones(1, 8, 8, dtype=half, device="cuda")
    y, kept = local.experts(x, r, w1, None, w2, None, "relu", keep=True)
    g = local.experts_backward(torch.ones_like(y), x, r, w1, None, w2, None, kept, "relu")
    assert (g.x[:, 1] == 4 * 8).all()
