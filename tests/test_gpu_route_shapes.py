"""Numbers of experts and groups at the edges of what routing takes."""
import pytest
import torch

from experts_util import route64
from operators_util import rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2104_08378_b200 import binding
    return binding


# Groups just wider than the lanes that look through them, so that rows of them in shared memory are furthest apart: the most of it that there are for 23 to 30
# groups and for 15; (1024, 32) and (660, 20) have less.
@pytest.mark.parametrize("E,groups", [(1020, 30), (1015, 29), (1008, 28), (972, 27), (988, 26), (1000, 25), (816, 24), (782, 23), (1012, 23), (1005, 15), (1024, 32), (660, 20)])
@pytest.mark.parametrize("group_score", ["max", "top2"])
def test_wide_groups(sp, E, groups, group_score):
    logits = rand((21, E), "f32", E, 1.5)
    for bias in (None, rand((E,), "f32", groups, 0.1)):
        how = dict(score="sigmoid", bias=bias, groups=groups, top_groups=5, group_score=group_score, scale=2.5)
        weights, experts = sp.route(logits, 8, **how)
        want_weights, want = route64(logits, 8, **how)
        assert torch.equal(experts, want)
        # (as in test_gpu_route.py: the exponential of a difference, the logarithm of the sigmoid, a sum and a division)
        assert bool(((weights.double() - want_weights).abs() <= 2.0 ** -17 * want_weights).all())


@pytest.mark.parametrize("how", [{"groups": 2 ** 32 + 1}, {"groups": 2 ** 32 + 4, "top_groups": 2}, {"groups": 4, "top_groups": 2 ** 32 + 2}, {"groups": -1}, {"groups": 4, "top_groups": 0},
                                 {"groups": 2 ** 70}])
def test_numbers_of_groups_that_do_not_fit_an_int(sp, how):
    with pytest.raises(sp.Sp24Error) as e:
        sp.route(rand((4, 64), "f32", 1), 2, **how)
    assert e.value.status == sp.ERR_SHAPE
