"""What the experts' operators refuse, before any device work: by the library's entry points and by the binding."""
import ctypes

import pytest
import torch

from paper_2104_08378_b200 import binding as sp

ONE, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4097)
F = ctypes.c_float


def route(t=sp.BF16, T=4, E=64, logits=ONE, ld=64, score=0, bias=ONE, groups=4, top=2, by=1, k=8, renorm=1, scale=1.0, weights=ONE, experts=ONE):
    return sp.lib.sp24_route(t, T, E, logits, ld, score, bias, groups, top, by, k, renorm, F(scale), weights, experts, None)


@pytest.mark.parametrize("status,args", [
    (2, {"t": sp.I8}), (3, {"T": -1}), (3, {"E": 0}), (3, {"E": 1025, "ld": 1025, "groups": 1, "top": 1}), (3, {"groups": 0}), (3, {"groups": 5}), (3, {"groups": 64}),
    (3, {"top": 0}), (3, {"top": 5}), (3, {"k": 0}), (3, {"k": 33}), (3, {"k": 17, "top": 1}), (6, {"score": 2}), (6, {"by": 2}), (6, {"score": -1}),
    (1, {"logits": None}), (1, {"weights": None}), (1, {"experts": None}), (4, {"ld": 63}), (5, {"logits": ODD}), (5, {"bias": ctypes.c_void_p(4098)}),
    (5, {"weights": ctypes.c_void_p(4098)}), (5, {"experts": ODD}), (0, {"T": 0, "logits": None})])
def test_route(status, args):
    assert route(**args) == status


def route_backward(t=sp.F32, T=4, E=64, dw=ONE, logits=ONE, ld=64, experts=ONE, k=8, score=0, out=ctypes.c_void_p(8192), ldd=64):
    return sp.lib.sp24_route_backward(t, T, E, dw, logits, ld, experts, k, score, 1, F(1.0), out, ldd, None)


@pytest.mark.parametrize("status,args", [
    (2, {"t": sp.E4M3}), (3, {"T": -1}), (3, {"E": 1025}), (3, {"k": 0}), (3, {"k": 33}), (6, {"score": 7}), (1, {"dw": None}), (1, {"logits": None}),
    (1, {"experts": None}), (1, {"out": None}), (4, {"ld": 1}), (4, {"ldd": 63}), (4, {"out": ONE, "ldd": 72}), (5, {"out": ctypes.c_void_p(8194)}),
    (5, {"dw": ODD}), (0, {"T": 0})])
def test_route_backward(status, args):
    assert route_backward(**args) == status


def order(slots=64, E=8, align=16, experts=ONE, offsets=ONE, position=ONE, source=ONE, ws=ONE, ws_bytes=1 << 20):
    return sp.lib.sp24_expert_order(slots, E, align, experts, offsets, position, source, ws, ws_bytes, None)


@pytest.mark.parametrize("status,args", [
    (3, {"slots": -1}), (3, {"E": 0}), (3, {"E": 1025}), (3, {"align": 0}), (3, {"align": 257}), (3, {"slots": 2 ** 31}), (3, {"slots": 2 ** 31 - 8}),
    (1, {"experts": None}), (1, {"offsets": None}), (1, {"position": None}), (1, {"source": None}), (5, {"offsets": ODD}), (5, {"source": ODD}),
    (1, {"slots": 0, "offsets": None}), (7, {"slots": 10 ** 6, "ws": None}), (7, {"slots": 10 ** 6, "ws_bytes": 64}), (7, {"slots": 10 ** 6, "ws": ctypes.c_void_p(4100)})])
def test_order(status, args):
    assert order(**args) == status


def test_rows_of_an_order():
    rows = sp.lib.sp24_expert_rows
    assert rows(64, 8, 1) == 64 and rows(64, 8, 16) == 64 + 8 * 15 + 8 and rows(3, 8, 16) == 48 and rows(0, 8, 16) == 0
    assert rows(-1, 8, 1) == rows(4, 0, 1) == rows(4, 8, 0) == 0 and rows(2 ** 31 - 8, 8, 16) >= 2 ** 31


def gather(t=sp.BF16, T=4, K=64, x=ONE, ldx=64, scale=ONE, k=2, position=ONE, rows=8, source=ONE, out=ctypes.c_void_p(8192), ldo=64, out_scale=ONE):
    return sp.lib.sp24_expert_gather(t, T, K, x, ldx, scale, k, position, rows, source, out, ldo, out_scale, None)


def combine(t=sp.BF16, T=4, K=64, rows=8, y=ONE, ldy=64, k=2, position=ONE, weights=ONE, residual=ONE, ldr=64, out=ctypes.c_void_p(8192), ldo=64):
    return sp.lib.sp24_expert_combine(t, T, K, rows, y, ldy, k, position, weights, residual, ldr, out, ldo, None)


def combine_backward(t=sp.BF16, T=4, K=64, rows=8, dout=ONE, lddo=64, y=ONE, ldy=64, k=2, position=ONE, source=ONE, weights=ONE, dy=ctypes.c_void_p(8192), lddy=64,
                     dw=ONE):
    return sp.lib.sp24_expert_combine_backward(t, T, K, rows, dout, lddo, y, ldy, k, position, source, weights, dy, lddy, dw, None)


SIZES = [(3, {"T": -1}), (3, {"K": 0}), (3, {"K": 2 ** 30 + 1}), (3, {"rows": -1}), (3, {"rows": 2 ** 31}), (3, {"k": 0}), (3, {"k": 33}), (1, {"position": None})]


@pytest.mark.parametrize("status,args", SIZES + [
    (2, {"t": 99}), (1, {"x": None}), (1, {"source": None}), (1, {"out": None}), (1, {"scale": None}), (1, {"out_scale": None}), (4, {"ldx": 63}), (4, {"ldo": 0}),
    (5, {"x": ODD}), (5, {"out": ODD}), (5, {"scale": ODD}), (0, {"rows": 0, "T": 0})])
def test_gather(status, args):
    assert gather(**args) == status


@pytest.mark.parametrize("status,args", SIZES + [
    (2, {"t": sp.I8}), (1, {"y": None}), (1, {"out": None}), (4, {"ldy": 63}), (4, {"ldr": 63}), (4, {"ldo": 63}), (4, {"out": ONE, "ldo": 72}), (5, {"y": ODD}),
    (5, {"residual": ODD}), (5, {"weights": ctypes.c_void_p(4098)}), (0, {"T": 0})])
def test_combine(status, args):
    assert combine(**args) == status


@pytest.mark.parametrize("status,args", SIZES + [
    (2, {"t": sp.E4M3}), (1, {"dout": None}), (1, {"y": None}), (1, {"source": None}), (1, {"weights": None}), (1, {"dy": None}), (1, {"dw": None}),
    (4, {"lddo": 63}), (4, {"ldy": 63}), (4, {"lddy": 63}), (4, {"dy": ONE, "lddy": 72}), (5, {"dy": ODD}), (5, {"dw": ODD}), (0, {"T": 0, "rows": 0})])
def test_combine_backward(status, args):
    assert combine_backward(**args) == status


def linear(ab=sp.BF16, cd=sp.BF16, E=4, M=64, K=64, rows=33, lda=32, ldx=64, ldd=64, ldr=64, ldp=64, dense=0, act=1, row_scale=ONE, col_scale=None, bias=ONE,
           residual=ONE, pre=ctypes.c_void_p(8192), A=ONE, meta=ONE, X=ONE, offsets=ONE, D=ctypes.c_void_p(12288), ws=ONE, ws_bytes=256):
    d = sp.ExpertDesc(ab, cd, E, M, K, rows, lda, ldx, ldd, ldr, ldp, dense)
    e = sp.ExpertEpilogue(row_scale, col_scale, bias, act, residual, pre)
    return sp.lib.sp24_expert_linear(ctypes.byref(d), ctypes.byref(e), A, meta, X, offsets, D, ws, ws_bytes, None)


@pytest.mark.parametrize("status,args", [
    (2, {"ab": sp.F32, "cd": sp.F32}), (2, {"ab": sp.I32}), (2, {"cd": sp.F16}), (2, {"ab": sp.I8, "cd": sp.I32}), (2, {"ab": sp.I8, "cd": sp.I8}), (6, {"act": 5}), (6, {"act": -1}),
    (6, {"col_scale": ONE}), (6, {"pre": ONE}), (6, {"pre": ctypes.c_void_p(12288)}), (3, {"E": 0}), (3, {"E": 1025}), (3, {"M": 40}), (3, {"K": 72}), (3, {"rows": -1}),
    (3, {"ab": sp.I8, "M": 48}), (3, {"M": 0}), (3, {"E": 1024, "M": 2 ** 21, "ldd": 2 ** 21, "ldr": 2 ** 21, "ldp": 2 ** 21}), (3, {"rows": 2 ** 30 + 1}),
    (1, {"A": None}), (1, {"meta": None}), (1, {"X": None}), (1, {"offsets": None}), (1, {"D": None}), (7, {"ws": None}), (7, {"ws_bytes": 255}),
    (7, {"ws": ctypes.c_void_p(4104)}), (4, {"lda": 24}), (4, {"lda": 36}), (4, {"ldx": 56}), (4, {"ldd": 56}), (4, {"ldd": 68}), (4, {"ldr": 56}), (4, {"ldp": 68}),
    (4, {"dense": 1}), (5, {"A": ctypes.c_void_p(4104)}), (5, {"X": ctypes.c_void_p(4104)}), (5, {"residual": ctypes.c_void_p(4104)}), (5, {"bias": ctypes.c_void_p(4098)}),
    (5, {"offsets": ctypes.c_void_p(4098)}), (0, {"rows": 0, "A": None})])
def test_linear(status, args):
    assert linear(**args) == status


def gradient(which, ab=sp.F16, cd=sp.F16, E=4, M=64, K=64, rows=48, lda=64, ldx=64, ldd=64, a=ONE, b=ONE, offsets=ONE, out=ONE, ws=ONE, ws_bytes=256):
    d = ctypes.byref(sp.ExpertDesc(ab, cd, E, M, K, rows, lda, ldx, ldd, 0, 0, 1))
    if which == "dx":
        return sp.lib.sp24_expert_linear_dx(d, a, b, offsets, out, ws, ws_bytes, None)
    return sp.lib.sp24_expert_linear_dw(d, a, b, offsets, None, out, ws, ws_bytes, None)


@pytest.mark.parametrize("which", ["dx", "dw"])
@pytest.mark.parametrize("status,args", [
    (2, {"ab": sp.I8, "cd": sp.I8}), (2, {"cd": sp.F32}), (3, {"E": 0}), (3, {"M": 24}), (3, {"K": 40}), (3, {"rows": -1}), (1, {"a": None}), (1, {"b": None}),
    (1, {"offsets": None}), (1, {"out": None}), (7, {"ws": None}), (7, {"ws_bytes": 8}), (4, {"lda": 56}), (4, {"ldx": 56}), (4, {"ldx": 68}), (5, {"a": ODD}),
    (5, {"b": ctypes.c_void_p(4104)}), (5, {"out": ctypes.c_void_p(4104)}), (5, {"offsets": ODD})])
def test_gradients(which, status, args):
    assert gradient(which, **args) == status


def test_gradients_own_strides():
    assert gradient("dx", ldd=56) == gradient("dx", ldd=68) == gradient("dw", ldd=56) == gradient("dw", ldd=68) == 4
    assert gradient("dx", rows=0, a=None) == 0


def act_backward(t=sp.BF16, act=3, E=4, M=64, rows=48, dy=ONE, lddy=64, z=ONE, ldz=64, offsets=ONE, dz=ONE, lddz=64, out=ONE, ws=ONE, ws_bytes=1 << 20):
    return sp.lib.sp24_expert_act_backward(t, act, E, M, rows, dy, lddy, z, ldz, offsets, dz, lddz, out, ws, ws_bytes, None)


@pytest.mark.parametrize("status,args", [
    (2, {"t": sp.I8}), (6, {"act": 9}), (3, {"E": 0}), (3, {"E": 1025}), (3, {"M": 0}), (3, {"rows": -1}), (1, {"dy": None}), (1, {"z": None}), (1, {"offsets": None}),
    (4, {"lddy": 63}), (4, {"ldz": 63}), (4, {"lddz": 63}), (5, {"dy": ODD}), (5, {"out": ODD}), (5, {"dz": ODD}), (7, {"ws": None}),
    (7, {"ws_bytes": 64}), (7, {"ws": ctypes.c_void_p(4104)}), (0, {"out": None, "dz": None})])
def test_act_backward(status, args):
    assert act_backward(**args) == status


def test_nothing_to_describe():
    assert sp.lib.sp24_expert_linear(None, None, None, None, None, None, None, None, 0, None) == 1
    assert sp.lib.sp24_expert_linear_dx(None, None, None, None, None, None, 0, None) == sp.lib.sp24_expert_linear_dw(None, None, None, None, None, None, None, 0, None) == 1


def refused(status, fn, *args, **kwargs):
    with pytest.raises(sp.Sp24Error) as e:
        fn(*args, **kwargs)
    assert e.value.status == status


def test_the_binding_takes_cuda_tensors_only():
    x, w, i = torch.zeros(4, 64), torch.zeros(4, 2), torch.zeros(4, 2, dtype=torch.int32)
    order_ = sp.ExpertOrder(torch.zeros(9, dtype=torch.int32), i, torch.zeros(8, dtype=torch.int32))
    refused(6, sp.route, x, 2)
    refused(2, sp.route, x.double(), 2)
    refused(3, sp.route, x[0], 2)
    refused(6, sp.route_backward, w, x, i)
    refused(6, sp.expert_order, i, 8)
    refused(3, sp.expert_order, i[0], 8)
    refused(6, sp.expert_gather, x, order_)
    refused(2, sp.expert_gather, x.double(), order_)
    refused(6, sp.expert_combine, x, order_, w)
    refused(6, sp.expert_combine_backward, x, x, order_, w)
    v = torch.zeros(2, 64, 32, dtype=torch.bfloat16)
    refused(6, sp.expert_compress, v)
    refused(2, sp.expert_compress, v.float())
    refused(6, sp.expert_linear, v, None, x.bfloat16(), torch.zeros(3, dtype=torch.int32))
    refused(2, sp.expert_linear, v.float(), None, x, torch.zeros(3, dtype=torch.int32))
    refused(6, sp.expert_linear_backward, x.bfloat16(), None, x.bfloat16(), v, torch.zeros(3, dtype=torch.int32))
    refused(2, sp.expert_linear_backward, x, None, x, v, torch.zeros(3, dtype=torch.int32))
