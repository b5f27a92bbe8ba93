"""The weights' gradient with its pattern in rows so long that their metadata are more than 2^31 bytes."""
import pytest
import torch

from operators_util import rand

pytestmark = pytest.mark.gpu


def test_pattern_behind_column_2_to_the_27():
    from paper_2104_08378_b200 import binding as sp
    if torch.cuda.mem_get_info()[0] < 24 * 2 ** 30:
        pytest.skip("needs 24 GiB")
    M, K, rows, tail = 16, 2 ** 27 + 512, 16, 1024
    X = torch.zeros((rows, K), dtype=torch.bfloat16, device="cuda")
    dy = rand((rows, M), "bf16", 1)
    X[:, -tail:] = rand((rows, tail), "bf16", 2)
    X[:, :tail] = rand((rows, tail), "bf16", 3)
    # the first and last 1024 columns have patterns of their own, the ones between keep what the metadata's zeros name
    patterns = [sp.prune(rand((M, tail), "bf16", seed)) for seed in (4, 5)]
    meta = torch.zeros((1, sp.meta_bytes("bf16", M, K)), dtype=torch.uint8, device="cuda")
    for at, W in zip((slice(0, sp.meta_bytes("bf16", M, tail)), slice(-sp.meta_bytes("bf16", M, tail), None)), patterns):
        meta[0, at] = sp.compress(W)[1].view(-1)
    dW = torch.empty((1, M, K), dtype=torch.bfloat16, device="cuda")
    desc = sp.ExpertDesc(sp.BF16, sp.BF16, 1, M, K, rows, K, K, M, 0, 0, 1)
    ws = sp.workspace(X.device)
    offsets = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    status = sp.lib.sp24_expert_linear_dw(desc, dy.data_ptr(), X.data_ptr(), offsets.data_ptr(), meta.data_ptr(), dW.data_ptr(), ws.data_ptr(), ws.numel(),
                                          torch.cuda.current_stream().cuda_stream)
    assert status == 0 and sp.gemm_status() == 0
    for at, W in zip((slice(0, tail), slice(-tail, None)), patterns):
        want = dy.double().T @ X[:, at].double() * (W != 0)
        # 16 products summed in FP32 (2^-19 of their magnitudes at most), rounded once to half a step
        bound = 2.0 ** -8 * want.abs() + 2.0 ** -18 * (dy.double().abs().T @ X[:, at].double().abs())
        assert bool(((dW[0, :, at].double() - want).abs() <= bound).all())
        assert bool((dW[0, :, at][W == 0] == 0).all())
