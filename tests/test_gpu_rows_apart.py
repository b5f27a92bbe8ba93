"""A row's norm depends on its values and on where it lies modulo 16 bytes, not on where the other rows lie: a row at a boundary by itself, and as one of a
matrix whose other rows lie between boundaries (which takes other loads, teams and, at the longest, another kernel)."""
import pytest
import torch

from operators_util import DTYPE, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2104_08378_b200 import binding
    return binding


@pytest.mark.parametrize("t,K", [("bf16", 64), ("bf16", 256), ("f16", 1024), ("bf16", 8192), ("bf16", 12288), ("f16", 12288), ("f16", 14336), ("bf16", 16384), ("f32", 2048), ("f32", 6144),
                                 ("f32", 8192)])
def test_rows_at_boundaries_among_others(sp, t, K):
    rows = 160
    x, r, w = rand((rows, K), t, 1, pad=5), rand((rows, K), t, 2, pad=5), rand((K,), t, 3)
    for residual in (None, r):
        for quant in (None, "i8", "e5m2"):
            out = torch.empty((rows, K + 5), dtype=DTYPE[quant or t], device="cuda")[:, :K]
            y, _, scale, rstd = sp.rms_norm(x, w, residual=residual, quant=quant, with_rstd=True, out=out)
            for i in range(0, rows, 16):
                assert x[i].data_ptr() % 16 == 0 and y[i].data_ptr() % 16 == 0
                one = sp.rms_norm(x[i:i + 1], w, residual=None if residual is None else residual[i:i + 1], quant=quant, with_rstd=True)
                assert torch.equal(one[3], rstd[i:i + 1]) and torch.equal(one[0].view(torch.uint8), y[i:i + 1].contiguous().view(torch.uint8))
                assert quant is None or torch.equal(one[2], scale[i:i + 1])
