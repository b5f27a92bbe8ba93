"""Results that lie over inputs which are read in another order: refused, before any device work, by the experts' operators."""
import ctypes

import pytest

from paper_2104_08378_b200 import binding as sp

BASE = 1 << 20
UNSUPPORTED = 6


def at(offset):
    return ctypes.c_void_p(BASE + offset)


FAR = at(1 << 18)


def gather(x, out, T=4, K=64, rows=8, ldx=64, ldo=64):
    return sp.lib.sp24_expert_gather(sp.BF16, T, K, x, ldx, None, 2, FAR, rows, FAR, out, ldo, None, None)


# (offsets in bytes; rows of 128 bytes)
@pytest.mark.parametrize("args", [
    {"x": at(0), "out": at(0)}, {"x": at(128), "out": at(0)}, {"x": at(0), "out": at(3 * 128 + 64)}, {"x": at(7 * 128), "out": at(0)}, {"x": at(2), "out": at(0)},
    {"x": at(0), "out": at(0), "T": 1, "rows": 1}, {"x": at(64), "out": at(0), "ldx": 128, "ldo": 128}, {"x": at(0), "out": at(1200), "ldx": 640},
    {"x": at(254), "out": at(0), "ldo": 128}])
def test_gather(args):
    assert gather(**args) == UNSUPPORTED


def combine(y, out, residual=None, T=4, rows=8, ldr=64):
    return sp.lib.sp24_expert_combine(sp.BF16, T, 64, rows, y, 64, 2, FAR, FAR, residual, ldr, out, 64, None)


@pytest.mark.parametrize("args", [
    {"y": at(0), "out": at(0)}, {"y": at(0), "out": at(0), "residual": at(0)}, {"y": at(0), "out": at(7 * 128)}, {"y": at(512), "out": at(128)},
    {"y": at(1 << 16), "out": at(0), "residual": at(128)}, {"y": at(1 << 16), "out": at(256), "residual": at(0)}, {"y": at(0), "out": at(0), "T": 1, "rows": 1}])
def test_combine(args):
    assert combine(**args) == UNSUPPORTED


def combine_backward(dout, y, dy, rows=8):
    return sp.lib.sp24_expert_combine_backward(sp.BF16, 4, 64, rows, dout, 64, y, 64, 2, FAR, FAR, FAR, dy, 64, FAR, None)


@pytest.mark.parametrize("args", [
    {"dout": at(0), "y": at(1 << 16), "dy": at(0)}, {"dout": at(1024 - 128), "y": at(1 << 16), "dy": at(0)}, {"dout": at(1 << 16), "y": at(0), "dy": at(128)},
    {"dout": at(1 << 16), "y": at(128), "dy": at(0)}, {"dout": at(0), "y": at(0), "dy": at(0)}])
def test_combine_backward(args):
    assert combine_backward(**args) == UNSUPPORTED


def act_backward(dy, z, dz, t=sp.BF16, act=3, M=64, lddz=64):
    return sp.lib.sp24_expert_act_backward(t, act, 4, M, 48, dy, 64, z, 64, FAR, dz, lddz, FAR, FAR, 1 << 20, None)


@pytest.mark.parametrize("args", [
    {"dy": at(0), "z": at(1 << 16), "dz": at(0)}, {"dy": at(1 << 16), "z": at(0), "dz": at(0)}, {"dy": at(0), "z": at(1 << 16), "dz": at(47 * 128)},
    {"dy": at(0), "z": None, "dz": at(0), "act": 0}, {"dy": at(256), "z": at(1 << 16), "dz": at(0), "t": sp.F32}, {"dy": at(0), "z": at(1 << 16), "dz": at(64), "M": 33},
    {"dy": at(0), "z": at(1 << 16), "dz": at(160), "lddz": 640}])
def test_act_backward(args):
    assert act_backward(**args) == UNSUPPORTED


# 4 experts, M = K = 64 in 16 bits: the weights' values are 16 KB (dense 32 KB), 33 rows of X, D, residual and pre a little more than 4 KB each
W_AT, X_AT, D_AT, R_AT, Z_AT = 0, 1 << 16, 2 << 16, 3 << 16, 5 << 16


def linear(A=W_AT, X=X_AT, D=D_AT, residual=None, pre=None, ldr=64, dense=0):
    d = sp.ExpertDesc(sp.BF16, sp.BF16, 4, 64, 64, 33, 64 if dense else 32, 64, 64, ldr, 64, dense)
    e = sp.ExpertEpilogue(None, None, None, 0, None if residual is None else at(residual), None if pre is None else at(pre))
    return sp.lib.sp24_expert_linear(ctypes.byref(d), ctypes.byref(e), at(A), FAR, at(X), FAR, at(D), at(7 << 16), 256, None)


@pytest.mark.parametrize("args", [
    {"D": X_AT}, {"D": X_AT + 32 * 128}, {"D": X_AT - 32 * 128}, {"D": W_AT}, {"D": W_AT + 16384 - 64}, {"D": W_AT + 32768 - 64, "dense": 1}, {"pre": X_AT}, {"pre": W_AT},
    {"pre": D_AT}, {"pre": D_AT + 128}, {"residual": R_AT, "pre": R_AT}, {"residual": R_AT, "pre": R_AT + 128}, {"residual": D_AT + 128}, {"residual": D_AT - 256}])
def test_linear(args):
    assert linear(**args) == UNSUPPORTED


def test_the_residual_that_is_the_result_has_its_rows():
    assert linear(residual=D_AT, ldr=72) == 4


def gradient(which, dz=X_AT, other=W_AT, out=D_AT):
    d = ctypes.byref(sp.ExpertDesc(sp.BF16, sp.BF16, 4, 64, 64, 48, 64, 64, 64, 0, 0, 1))
    if which == "dx":
        return sp.lib.sp24_expert_linear_dx(d, at(dz), at(other), FAR, at(out), at(7 << 16), 256, None)
    return sp.lib.sp24_expert_linear_dw(d, at(dz), at(other), FAR, None, at(out), at(7 << 16), 256, None)


@pytest.mark.parametrize("which,args", [
    ("dx", {"out": X_AT}), ("dx", {"out": X_AT + 47 * 128}), ("dx", {"out": W_AT}), ("dx", {"out": 255 * 128}), ("dw", {"out": X_AT}), ("dw", {"out": X_AT - 255 * 128}),
    ("dw", {"out": W_AT + 47 * 128}), ("dw", {"out": W_AT})])
def test_gradients(which, args):
    assert gradient(which, **args) == UNSUPPORTED


@pytest.mark.parametrize("logits,out,T,ld", [(0, 256, 4, 64), (3 * 256, 0, 4, 64), (0, 4, 4, 64), (0, 4, 1, 64), (0, 252, 4, 128), (508, 0, 4, 128)])
def test_route_backward(logits, out, T, ld):
    assert sp.lib.sp24_route_backward(sp.F32, T, 64, FAR, at(logits), ld, FAR, 8, 0, 1, ctypes.c_float(1.0), at(out), ld, None) == UNSUPPORTED
