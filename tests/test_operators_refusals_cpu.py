"""What the operators around the products refuse, before any device work: by the library's entry points and by the binding."""
import ctypes

import pytest
import torch

from paper_2104_08378_b200 import binding as sp

ONE = ctypes.c_void_p(4096)
F = ctypes.c_float


def norm(t=sp.BF16, rows=4, K=64, x=ONE, ldx=64, r=ONE, ldr=64, w=ONE, wt=sp.BF16, eps=1e-6, h=ctypes.c_void_p(8192), ldh=64, out=sp.BF16, y=ONE,
         ldy=64, scale=ONE, rstd=ONE):
    return sp.lib.sp24_rms_norm(t, rows, K, x, ldx, r, ldr, w, wt, F(eps), h, ldh, out, y, ldy, scale, rstd, None)


@pytest.mark.parametrize("status,args", [
    (2, {"t": sp.I8}), (2, {"t": sp.I32}), (2, {"out": sp.F16}), (2, {"out": sp.I32}), (2, {"wt": sp.F16}), (2, {"t": 99}),
    (3, {"rows": -1}), (3, {"K": 0}), (3, {"K": 2 ** 30 + 1}),
    (6, {"eps": -1.0}), (6, {"h": ONE}), (6, {"eps": float("nan")}), (6, {"r": None}),
    (1, {"x": None}), (1, {"y": None}), (1, {"out": sp.I8, "scale": None}),
    (4, {"ldx": 63}), (4, {"ldr": 63}), (4, {"ldh": 0}), (4, {"ldy": -64}),
    (5, {"x": ctypes.c_void_p(4097)}), (5, {"w": ctypes.c_void_p(4098), "wt": sp.F32}), (5, {"rstd": ctypes.c_void_p(4098)}),
    (0, {"rows": 0, "x": None, "y": None})])
def test_norm(status, args):
    assert norm(**args) == status


def norm_backward(t=sp.BF16, rows=4, K=64, dy=ONE, lddy=64, h=ONE, ldh=64, w=ONE, wt=sp.BF16, rstd=ONE, dh=ONE, lddh=64, dx=ONE,
                  lddx=64, dw=ONE, ws=ONE, ws_bytes=1 << 20):
    return sp.lib.sp24_rms_norm_backward(t, rows, K, dy, lddy, h, ldh, w, wt, rstd, dh, lddh, dx, lddx, dw, ws, ws_bytes, None)


@pytest.mark.parametrize("status,args", [
    (2, {"t": sp.E4M3}), (2, {"wt": sp.F16}), (3, {"rows": -1}), (3, {"K": 0}), (1, {"dy": None}), (1, {"h": None}),
    (1, {"rstd": None}), (1, {"dx": None}), (4, {"lddy": 63}), (4, {"ldh": 63}), (4, {"lddh": 63}), (4, {"lddx": 63}),
    (5, {"dx": ctypes.c_void_p(4097)}), (7, {"ws": None}), (7, {"ws_bytes": 4 * 64 * 4 - 1}), (7, {"ws": ctypes.c_void_p(4100)}),
    (0, {"rows": 0, "dw": None})])
def test_norm_backward(status, args):
    assert norm_backward(**args) == status


def test_workspace_of_the_norms_gradient():
    size = sp.lib.sp24_rms_norm_backward_workspace_bytes
    assert size(4, 64) == 4 * 64 * 4 and size(10 ** 6, 64) == size(2 * 10 ** 6, 64) and size(0, 64) == size(4, 0) == 0


def refused(status, fn, *args, **kwargs):
    with pytest.raises(sp.Sp24Error) as e:
        fn(*args, **kwargs)
    assert e.value.status == status


def test_the_binding_takes_cuda_tensors_only():
    x, w, r = torch.zeros(4, 64), torch.zeros(64), torch.zeros(4)
    refused(6, sp.rms_norm, x, w)
    refused(6, sp.rms_norm_backward, x, x, w, r)
    refused(2, sp.rms_norm, x.to(torch.int8))
    refused(2, sp.rms_norm, x.double())
    refused(3, sp.rms_norm, x[0])
    refused(6, sp.gated_act, x, x)
    refused(6, sp.gated_act, x, act="tanh")
    refused(6, sp.gated_act_backward, x, x, x)
    refused(6, sp.act_backward, x, x, act="gelu")


def gated(t=sp.BF16, act=3, rows=4, F=64, g=ONE, ldg=64, u=ONE, ldu=64, out=sp.BF16, y=ONE, ldy=64, scale=ONE):
    return sp.lib.sp24_gated_act(t, act, rows, F, g, ldg, u, ldu, out, y, ldy, scale, None)


def gated_backward(t=sp.BF16, act=3, rows=4, F=64, dy=ONE, lddy=64, g=ONE, ldg=64, u=ONE, ldu=64, dg=ONE, lddg=64, du=ctypes.c_void_p(8192), lddu=64):
    return sp.lib.sp24_gated_act_backward(t, act, rows, F, dy, lddy, g, ldg, u, ldu, dg, lddg, du, lddu, None)


def act_backward(t=sp.BF16, act=3, rows=4, cols=64, dy=ONE, lddy=64, z=ONE, ldz=64, dz=ONE, lddz=64, dzt=ONE, lddzt=4, db=ONE, over_rows=1,
                 ws=ONE, ws_bytes=1 << 20):
    return sp.lib.sp24_act_backward(t, act, rows, cols, dy, lddy, z, ldz, dz, lddz, dzt, lddzt, db, over_rows, ws, ws_bytes, None)


@pytest.mark.parametrize("status,args", [
    (2, {"t": sp.I8}), (2, {"out": sp.F32}), (6, {"act": 5}), (6, {"act": -1}), (3, {"rows": -1}), (3, {"F": 0}), (1, {"g": None}),
    (1, {"y": None}), (1, {"out": sp.E4M3, "scale": None}), (4, {"ldg": 63}), (4, {"ldu": 63}), (4, {"ldy": 0}),
    (5, {"u": ctypes.c_void_p(4097)}), (0, {"rows": 0})])
def test_gated(status, args):
    assert gated(**args) == status


@pytest.mark.parametrize("status,args", [
    (2, {"t": sp.I32}), (6, {"act": 9}), (6, {"u": None}), (6, {"du": ONE}), (3, {"F": 0}), (1, {"dy": None}), (1, {"g": None}), (1, {"dg": None}),
    (1, {"du": None}), (4, {"lddy": 1}), (4, {"ldg": 1}), (4, {"ldu": 1}), (4, {"lddg": 1}), (4, {"lddu": 1}),
    (5, {"dg": ctypes.c_void_p(4097)}), (0, {"rows": 0})])
def test_gated_backward(status, args):
    assert gated_backward(**args) == status


@pytest.mark.parametrize("status,args", [
    (2, {"t": sp.I8}), (6, {"act": 9}), (3, {"rows": -1}), (3, {"cols": 2 ** 30 + 1}), (1, {"dy": None}), (1, {"z": None}),
    (4, {"lddy": 63}), (4, {"ldz": 63}), (4, {"lddz": 63}), (4, {"lddzt": 3}), (5, {"dzt": ctypes.c_void_p(4097)}),
    (5, {"db": ctypes.c_void_p(4098)}), (7, {"ws": None}), (7, {"ws_bytes": 255}), (0, {"rows": 0, "db": None}),
    (0, {"dz": None, "dzt": None, "db": None})])
def test_act_backward(status, args):
    assert act_backward(**args) == status


def linear(ab=sp.BF16, cd=sp.BF16, M=64, N=32, K=64, lda=32, ldb=64, ldc=32, ldd=32, order=0, dense=0, act=1, row_scale=ONE, col_scale=None, bias=ONE,
           residual=ONE, pre=ctypes.c_void_p(8192), ld_pre=32, A=ONE, meta=ONE, B=ONE, D=ctypes.c_void_p(12288), ws=ONE, ws_bytes=256):
    d = sp.GemmDesc(ab, cd, M, N, K, lda, ldb, ldc, ldd, sp.COL_MAJOR, 0, order, dense)
    e = sp.LinearEpilogue(row_scale, col_scale, bias, act, residual, pre, ld_pre)
    return sp.lib.sp24_linear(ctypes.byref(d), ctypes.byref(e), A, meta, B, D, ws, ws_bytes, None)


@pytest.mark.parametrize("status,args", [
    (2, {"ab": sp.I32}), (2, {"cd": sp.F16}), (2, {"ab": sp.I8, "cd": sp.I32}), (2, {"ab": sp.I8, "cd": sp.I8}), (2, {"ab": sp.E4M3, "cd": sp.I32}),
    (6, {"ab": sp.F32, "cd": sp.F16}), (6, {"act": 7}), (6, {"pre": ONE}), (6, {"pre": ctypes.c_void_p(12288)}), (6, {"act": -1}), (6, {"col_scale": ONE}), (6, {"order": 1, "ldd": 64}), (6, {"order": 3}),
    (3, {"M": 40}), (3, {"N": 24}), (3, {"K": 72}), (3, {"ab": sp.I8, "M": 48}), (3, {"M": -16}),
    (1, {"A": None}), (1, {"meta": None}), (1, {"B": None}), (1, {"D": None}), (7, {"ws": None}), (7, {"ws_bytes": 255}),
    (4, {"lda": 24}), (4, {"ldb": 56}), (4, {"ldc": 24}), (4, {"ldd": 36}), (4, {"ld_pre": 24}), (4, {"ld_pre": 36}),
    (5, {"residual": ctypes.c_void_p(4104)}), (5, {"pre": ctypes.c_void_p(4104)}), (5, {"bias": ctypes.c_void_p(4098)}),
    (5, {"row_scale": ctypes.c_void_p(4098)}), (0, {"N": 0})])
def test_linear(status, args):
    assert linear(**args) == status


def test_linear_without_a_problem():
    assert sp.lib.sp24_linear(None, None, None, None, None, None, None, 0, None) == 1
    x, w, m = torch.zeros(32, 64, dtype=torch.bfloat16), torch.zeros(64, 32, dtype=torch.bfloat16), torch.zeros(4096, dtype=torch.uint8)
    refused(6, sp.linear, w, m, x)
    refused(6, sp.linear_backward, x, x, x, w)


def test_calls_are_made_with_the_tensors_device_current(monkeypatch):
    """By position or by name, and not where it is current already; a stand-in for a tensor on a second device."""
    import contextlib
    import types
    made = []

    @contextlib.contextmanager
    def device(d):
        made.append(d)
        yield
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "device", device)
    call = sp._on_device_of("x")(lambda x, y=1: (x.device, y))
    there, here = (types.SimpleNamespace(is_cuda=True, device=f"cuda:{i}", get_device=lambda i=i: i) for i in (1, 0))
    assert call(there, y=2) == ("cuda:1", 2) and call(x=there) == ("cuda:1", 1) and made == ["cuda:1", "cuda:1"]
    assert call(here) == ("cuda:0", 1) and len(made) == 2
