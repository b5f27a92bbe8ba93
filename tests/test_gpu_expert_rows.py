"""Rows gathered in the experts' order and summed back, and their gradients, against plain implementations in 64 bits."""
import pytest
import torch

from experts_util import choice
from operators_util import DTYPE, close, rand

pytestmark = pytest.mark.gpu
SHAPES = [(1, 1, 1, 1), (1, 4096, 8, 8), (5, 64, 4, 2), (33, 520, 9, 3), (130, 75, 33, 5), (7, 1531, 6, 6), (3, 20000, 5, 2), (600, 256, 64, 8)]


@pytest.fixture(scope="module")
def sp():
    from paper_2104_08378_b200 import binding
    return binding


def rows_at(x, index):
    """x's rows, zeros where the index is negative."""
    return x.double()[index.clamp(min=0).long()] * (index >= 0)[..., None]


@pytest.mark.parametrize("t", ["bf16", "f16", "f32", "i8", "e4m3", "e5m2"])
@pytest.mark.parametrize("T,K,E,k", SHAPES)
@pytest.mark.parametrize("align", [1, 16])
def test_gather(sp, t, T, K, E, k, align):
    for pad, dropped in ((0, 0.0), (3, 0.3), (16, 0.3)):
        x = (rand((T, K), "f32", 1) * 20).to(DTYPE[t]) if t == "i8" else rand((T, K + pad), "f32", 1).to(DTYPE[t])[:, :K]
        order = sp.expert_order(choice(T, E, k, T + K, dropped), E, align=align)
        rows, source = order.source.shape[0], order.source
        out = torch.ones((rows, K + pad), dtype=torch.float32, device="cuda").to(DTYPE[t])[:, :K] if pad else None
        scale = rand((T,), "f32", 2)
        got, scales = sp.expert_gather(x, order, scale=scale, out=out)
        token = torch.where(source >= 0, source // k, source)
        assert got.dtype == DTYPE[t] and (out is None or got is out)
        assert torch.equal(got.double(), rows_at(x, token)) and torch.equal(scales, rows_at(scale[:, None], token)[:, 0].float())
        assert sp.expert_gather(x, order)[1] is None


# A sum of k + 1 products in FP32: k + 1 roundings of at most 2^-24 of the sum of the magnitudes each.
@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,K,E,k", SHAPES)
def test_combine(sp, t, T, K, E, k):
    for align, pad, dropped, weighted, residual in ((1, 0, 0.0, True, False), (16, 0, 0.3, True, True), (1, 5, 0.3, False, True), (16, 8, 0.3, False, False)):
        order = sp.expert_order(choice(T, E, k, T + K, dropped), E, align=align)
        y = rand((order.source.shape[0], K), t, 1, pad=pad)
        w = rand((T, k), "f32", 2) if weighted else None
        r = rand((T, K), t, 3, pad=pad) if residual else None
        parts = rows_at(y, order.position) * (1 if w is None else w.double()[:, :, None])
        want = parts.sum(1) + (0 if r is None else r.double())
        bound = (k + 2) * 2.0 ** -24 * (parts.abs().sum(1) + (0 if r is None else r.double().abs()))
        y[order.source < 0] = float("nan")            # rows that no slot has are not read
        got = sp.expert_combine(y, order, w, residual=r)
        close(got, want, t, bound)
        if residual:
            there = r.clone() if pad == 0 else r
            assert sp.expert_combine(y, order, w, residual=there, out=there) is there and torch.equal(there, got)


# dweights: chains of at most K / 2 + 16 additions of products (threads of a block, or elements of a vector).
@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,K,E,k", SHAPES)
def test_combine_backward(sp, t, T, K, E, k):
    for align, pad, dropped in ((1, 0, 0.0), (16, 0, 0.3), (16, 3, 0.3)):
        order = sp.expert_order(choice(T, E, k, T + K, dropped), E, align=align)
        y, dout = rand((order.source.shape[0], K), t, 1, pad=pad), rand((T, K), t, 2, pad=pad)
        w = rand((T, k), "f32", 3)
        used = order.source >= 0
        slot = order.source.clamp(min=0).long()
        want = dout.double()[slot // k] * (w.double().view(-1)[slot] * used)[:, None]
        products = rows_at(y, order.position) * dout.double()[:, None]
        y[~used] = float("nan")
        dy, dw = sp.expert_combine_backward(dout, y, order, w)
        close(dy, want, t, 0.0)
        close(dw, products.sum(2), "f32", (K / 2 + 16) * 2.0 ** -24 * products.abs().sum(2))
        if pad == 0:
            there = y.clone()
            again = sp.expert_combine_backward(dout, there, order, w, out=there)
            assert again[0] is there and torch.equal(there, dy) and torch.equal(again[1], dw)


def test_an_infinite_row_stays_with_its_tokens(sp):
    """Dropped slots count for nothing, whatever their weight; a weight of zero is a factor."""
    experts = torch.tensor([[0, 1], [1, -1], [-1, -1]], dtype=torch.int32, device="cuda")
    order = sp.expert_order(experts, 2)
    y = torch.ones((6, 64), device="cuda")
    y[3:] = float("inf")
    w = torch.tensor([[2.0, 3.0], [4.0, float("nan")], [float("inf"), 1.0]], device="cuda")
    got = sp.expert_combine(y, order, w)
    assert bool((got[0] == 5).all()) and bool((got[1] == 4).all()) and bool((got[2] == 0).all())


def test_positions_out_of_range_are_left_out(sp):
    """As a position may be that does not come from expert_order: refused by the kernels' own check."""
    order = sp.expert_order(choice(4, 3, 2, 1), 3)
    bad = order._replace(position=torch.where(order.position == 3, torch.full_like(order.position, 1000), order.position))
    x = rand((4, 64), "bf16", 1)
    there = torch.full((8, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    sp.expert_gather(x, bad, out=there)
    assert bool((there[3] == 9).all())
    y, w = rand((8, 64), "bf16", 2), rand((4, 2), "f32", 3)
    want = sp.expert_combine(y, order._replace(position=torch.where(order.position == 3, torch.full_like(order.position, -1), order.position)), w)
    assert torch.equal(sp.expert_combine(y, bad, w), want)
    _, dw = sp.expert_combine_backward(x, y, bad, w)
    assert bool((dw[order.position == 3] == 0).all())
