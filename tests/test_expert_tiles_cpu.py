"""Forced tiles that the experts' products do not have: refused before any device work."""
import ctypes

import pytest

from paper_2104_08378_b200 import binding as sp

ONE = ctypes.c_void_p(4096)


@pytest.fixture(autouse=True)
def automatic():
    yield
    sp.set_tile_override(None)


def linear(dense):
    d = sp.ExpertDesc(sp.BF16, sp.BF16, 4, 64, 64, 33, 64 if dense else 32, 64, 64, 64, 64, dense)
    e = sp.ExpertEpilogue(None, None, None, 0, None, None)
    return sp.lib.sp24_expert_linear(ctypes.byref(d), ctypes.byref(e), ONE, ONE, ctypes.c_void_p(65536), ONE, ctypes.c_void_p(131072), ONE, 256, None)


def dx():
    d = sp.ExpertDesc(sp.BF16, sp.BF16, 4, 64, 64, 48, 64, 64, 64, 0, 0, 1)
    return sp.lib.sp24_expert_linear_dx(ctypes.byref(d), ONE, ctypes.c_void_p(65536), ONE, ctypes.c_void_p(131072), ONE, 256, None)


@pytest.mark.parametrize("call", [lambda: linear(0), lambda: linear(1), dx])
@pytest.mark.parametrize("tile", ["1x0x1", "2x0x1", "1x31x1", "1x48x1", "1x160x1", "2x288x1", "1x64x2", "2x128x3", "3x64x1"])
def test_refused(call, tile):
    sp.set_tile_override(tile)
    assert call() == sp.ERR_UNSUPPORTED


def test_sparse_operands_end_at_224_columns():
    sp.set_tile_override("2x256x1")
    assert linear(0) == sp.ERR_UNSUPPORTED
