"""Results beside their inputs in one matrix, which share no byte with them, and those that are refused by both forms of the binding."""
import pytest
import torch

from experts_util import choice
from operators_util import rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2104_08378_b200 import binding
    return binding


def refused(sp, fn, *args, **kwargs):
    with pytest.raises(sp.Sp24Error) as e:
        fn(*args, **kwargs)
    assert e.value.status == sp.ERR_UNSUPPORTED


@pytest.mark.parametrize("T,K", [(1, 64), (40, 64), (40, 75)])
def test_rows_side_by_side(sp, T, K):
    order = sp.expert_order(choice(T, 5, 1, 1), 5)
    wide = rand((T, 2 * K), "bf16", 2)
    x, out = wide[:, :K], wide[:, K:]
    want = sp.expert_gather(x.clone(), order)[0]
    assert torch.equal(sp.expert_gather(x, order, out=out)[0], want)
    weights = rand((T, 1), "f32", 3)
    want = sp.expert_combine(out.clone(), order, weights)
    sp.expert_combine(out, order, weights, out=x)
    assert torch.equal(x, want)
    y = rand((T, K), "bf16", 4)
    want = sp.expert_combine_backward(x.clone(), y, order, weights)
    got = sp.expert_combine_backward(x, y, order, weights, out=out)
    assert torch.equal(out, want[0])
    # A sum's order goes by where the rows lie: chains of at most K / 2 + 16 additions on both sides, of half a step of FP32 (2^-24) each.
    products = x.double() * y.double()[order.position[:, 0].long()]
    assert bool(((got[1] - want[1]).double().abs()[:, 0] <= 2 * (K / 2 + 16) * 2.0 ** -24 * products.abs().sum(1)).all())


def test_rows_over_their_inputs(sp):
    order = sp.expert_order(choice(40, 5, 1, 1), 5)
    x, y, weights = rand((41, 64), "bf16", 2), rand((40, 64), "bf16", 3), rand((40, 1), "f32", 4)
    for name in ("gather", "combine", "combine_backward"):
        for out in (x[:40], x[1:]):
            if name == "gather":
                refused(sp, sp.expert_gather, x[:40], order, out=out)
            elif name == "combine":
                refused(sp, sp.expert_combine, x[:40], order, weights, out=out)
                if out.data_ptr() != x.data_ptr():
                    refused(sp, sp.expert_combine, y, order, weights, residual=x[:40], out=out)
            else:
                refused(sp, sp.expert_combine_backward, x[:40], y, order, weights, out=out)


def test_products_beside_and_over_their_operands(sp):
    """D and pre beside X in one matrix; over it, and a residual a row further on, refused."""
    E, M, K, rows = 3, 64, 64, 50
    A, meta = sp.expert_compress(rand((E, M, K), "bf16", 1))
    wide, offsets = rand((rows + 1, 4 * K), "bf16", 2), torch.tensor([0, 20, 20, 50], dtype=torch.int32, device="cuda")
    X, D, Z, R = (wide[:rows, i * K:(i + 1) * K] for i in range(4))
    want = sp.expert_linear(A, meta, X.clone(), offsets, act="silu", residual=R.clone(), pre=True)
    got = sp.expert_linear(A, meta, X, offsets, act="silu", residual=R, pre=Z, out=D)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and got[0] is D
    refused(sp, sp.expert_linear, A, meta, X, offsets, out=X)
    refused(sp, sp.expert_linear, A, meta, X, offsets, pre=X)
    refused(sp, sp.expert_linear, A, meta, X, offsets, residual=wide[1:, :K], out=wide[:rows, :K])
    refused(sp, sp.expert_linear, A, meta, X, offsets, residual=wide[1:, K:2 * K], out=D)


@pytest.mark.parametrize("E", [64, 65])
def test_logits_and_their_gradient_side_by_side(sp, E):
    wide = rand((41, 2 * E), "f32", 1)
    logits, out = wide[:40, :E], wide[:40, E:]
    g, experts = rand((40, 3), "f32", 2), choice(40, E, 3, 3)
    want = sp.route_backward(g, logits.clone(), experts)
    assert sp.route_backward(g, logits, experts, out=out) is out and torch.equal(out, want)
    refused(sp, sp.route_backward, g, logits, experts, out=wide[1:, :E])
