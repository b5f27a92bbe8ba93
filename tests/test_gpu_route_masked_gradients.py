"""The routing's gradient for tokens whose masks leave some experts, fewer than are chosen, or none."""
import math

import pytest
import torch

from operators_util import DTYPE, close, rand
from test_gpu_route import gradient64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("E,k,pad", [(64, 8, 0), (64, 8, 1), (256, 4, 0), (40, 3, 0), (600, 20, 0)])
def test_masked_tokens(t, score, renorm, E, k, pad):
    from paper_2104_08378_b200 import binding as sp
    logits = rand((48, E), t, E, 1.5, pad=pad)
    gone = torch.rand((48, E), generator=torch.Generator(device="cuda").manual_seed(k), device="cuda") < 0.5
    gone[8:16, 2:], gone[16:24, 1:], gone[24:32] = True, True, True      # (two experts at most, one, none)
    logits[gone] = -math.inf
    g = rand((48, k), "f32", 4)
    _, experts = sp.route(logits, k, score=score, renorm=renorm)
    assert bool((experts[24:32] == -1).all())
    got = sp.route_backward(g, logits, experts, score=score, renorm=renorm, scale=2.5)
    want = gradient64(g, logits, experts, score, renorm, 2.5)
    assert got.dtype == DTYPE[t] and bool((got[24:32] == 0).all()) and bool((got[gone] == 0).all())
    # scores off by 2^-18, differences of the g of up to the largest |g| of the token (as in test_gpu_route.py)
    close(got, want, t, 2.0 ** -15 * 2.5 * g.double().abs().amax(1, keepdim=True))
