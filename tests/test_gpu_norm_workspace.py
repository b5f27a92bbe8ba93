"""The workspace of the norm's gradient: a row for each block that there can be, and no more."""
import pytest
import torch

from operators_util import close, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2104_08378_b200 import binding
    return binding


@pytest.mark.parametrize("rows,K", [(100, 264), (148, 1032), (5000, 64), (700, 4096), (2000, 16384), (400, 20000)])
def test_size_and_what_is_behind_it(sp, rows, K):
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    size = sp.lib.sp24_rms_norm_backward_workspace_bytes(rows, K)
    assert size == min(rows, sms) * K * 4
    dy, h, rstd = rand((rows, K), "bf16", 1), rand((rows, K), "bf16", 2), rand((rows,), "f32", 3).abs() + 0.5
    dx, dw, ws = torch.empty_like(dy), torch.empty(K, device="cuda"), torch.full((size // 4 + 4096,), 7.0, device="cuda")
    args = [p.data_ptr() for p in (dy, h, rstd, dx, dw, ws)]

    def call(bytes_):
        return sp.lib.sp24_rms_norm_backward(sp.BF16, rows, K, args[0], K, args[1], K, None, sp.F32, args[2], None, K, args[3], K, args[4], args[5], bytes_,
                                             torch.cuda.current_stream().cuda_stream)
    assert call(size - 1) == 7 and call(size) == 0
    each = dy.double() * h.double() * rstd.double()[:, None]
    # (a chain of additions is at most 35 rows of a block, 15 teams of it and 148 blocks long, of 2^-24 of what it has summed)
    close(dw, each.sum(0), "f32", 2.0 ** -16 * each.abs().sum(0))
    assert bool((ws[size // 4:] == 7).all())
