"""Gradients of the linear layer: forms and arguments that go other ways through act_backward and linear_backward."""
import pytest
import torch

from operators_util import close, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2104_08378_b200 import binding
    return binding


class Silent:
    """A native part that leaves every call to the Python forms."""
    def __getattr__(self, name):
        return lambda *args: None


@pytest.fixture(params=["native", "python"])
def either(sp, request, monkeypatch):
    """The binding with its native calls and with its Python forms."""
    if request.param == "python":
        monkeypatch.setattr(sp, "_native", Silent())
    return sp


@pytest.mark.parametrize("t", ["f16", "bf16", "f32"])
def test_a_result_is_written_without_an_activation(either, t):
    for rows, cols, pad in ((48, 160, 0), (33, 75, 3), (1, 1, 0)):
        dy = rand((rows, cols), t, 1, pad=pad)
        out = torch.full_like(dy, 7.0)
        dz, dzt, db = either.act_backward(dy, None, act=None, cd_col_major=True, out=out)
        assert dz is out and torch.equal(out, dy) and torch.equal(dzt, dy.T)
        close(db, dy.double().sum(0), "f32", 2.0 ** -18 * dy.double().abs().sum(0))   # (chains of fewer than 64 additions)
        kept = dy.clone()
        dz, none, no_bias = either.act_backward(dy, None, act=None, transposed=False, bias=False, out=dy)
        assert dz is dy and none is None and no_bias is None and torch.equal(dy, kept)
        assert either.act_backward(dy, None, act=None)[0] is dy
        for wrong in (torch.empty((rows, cols + 1), dtype=dy.dtype, device="cuda"), torch.empty((rows, cols), dtype=torch.float64, device="cuda")):
            with pytest.raises(either.Sp24Error):
                either.act_backward(dy, None, act=None, out=wrong)


@pytest.mark.parametrize("t", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("act", [None, "silu"])
@pytest.mark.parametrize("cols", [True, False])
def test_the_results_gradient_may_lie_anywhere(either, t, act, cols):
    """The same gradients from dy in rows between 16-byte boundaries, and behind one, as from a packed dy."""
    M, N, K = 96, 48, 64
    W, X, dy = rand((M, K), t, 2), rand((N, K), t, 3), rand((N, M) if cols else (M, N), t, 4)
    pre = rand(dy.shape, t, 5)
    want = either.linear_backward(dy, pre, X, W, act=act, cd_col_major=cols)
    for pad, offset in ((3, 0), (16, 1), (0, 1)):
        room = torch.empty(dy.shape[0] * (dy.shape[1] + pad) + offset, dtype=dy.dtype, device="cuda")[offset:]
        there = room.as_strided(dy.shape, (dy.shape[1] + pad, 1))
        there.copy_(dy)
        got = either.linear_backward(there, pre, X, W, act=act, cd_col_major=cols)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(there, dy)
        # (its sums go through tiles in another order: chains of fewer than 64 additions)
        close(got[2], want[2].double(), "f32", 2.0 ** -17 * dy.double().abs().sum(0 if cols else 1))
