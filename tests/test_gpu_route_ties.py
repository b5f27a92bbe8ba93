"""Routing under a bias where the last place goes to one of two equal experts and a third is a little larger than both: what FP32 takes for a tie that the
index decides is none."""
import pytest
import torch

from experts_util import route64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2104_08378_b200 import binding
    return binding


def rows_with_ties(E, score, ahead, equal, seed):
    """(logits, bias): `ahead` experts that are clearly chosen, `equal` ones of the same logit and bias, behind them in the row one whose score is larger by
    less than FP32 sums with the bias show, and all others far behind.  At random places, in this order."""
    g = torch.Generator().manual_seed(seed)
    at = torch.randperm(E - 1, generator=g)[:ahead + equal + 1].sort().values + 1
    logits, bias = torch.zeros((3, E), device="cuda"), torch.full((E,), -1.0, device="cuda")
    logits[:, 0], bias[0] = 3.0, -3.0                # (softmax: what the others are small beside; never chosen)
    bias[at] = 0.5
    low = -16.0 if score == "softmax" else -20.0     # scores below 6e-9 beside 0.5, of which half a step is 3e-8
    logits[:, at[:ahead]] = torch.arange(ahead, device="cuda") * 0.25 - 1.0
    logits[:, at[ahead:]] = low
    logits[:, at[-1]] = low + 0.0625
    return logits, bias


@pytest.mark.parametrize("E", [12, 40, 64, 128, 256, 600])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("ahead,equal", [(0, 2), (1, 2), (2, 3), (3, 4)])
def test_a_larger_score_behind_equal_ones(sp, score, E, ahead, equal):
    for seed in range(6):
        logits, bias = rows_with_ties(E, score, ahead, equal, seed)
        for k in range(max(1, ahead), ahead + equal + 1):      # the last place before the equal ones and among them
            for groups in (1, 2):
                if k > E // groups:
                    continue
                how = dict(score=score, bias=bias, groups=groups, top_groups=groups, group_score="top2")
                want = route64(logits, k, **how)[1]
                assert torch.equal(sp.route(logits, k, **how)[1], want), (seed, k, groups)
                between = torch.nn.functional.pad(logits, (0, 1))[:, :E]   # (rows between boundaries)
                assert torch.equal(sp.route(between, k, **how)[1], want), (seed, k, groups)
