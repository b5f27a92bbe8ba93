"""The operators around the products through the binding's native calls and through its Python forms: the same results, types and
refusals, and outputs that stay inside their tensors."""
import pytest
import torch

from operators_util import HALF_STEP, TINY, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2104_08378_b200 import binding
    return binding


class Silent:
    """A native part that leaves every call to the Python forms."""
    def __getattr__(self, name):
        return lambda *args: None


def flat(result):
    return list(result) if isinstance(result, tuple) else [result]


def calls(sp):
    x, r, w, dy = rand((9, 520), "bf16", 1), rand((9, 520), "bf16", 2), rand((520,), "bf16", 3), rand((9, 520), "bf16", 4)
    w32, rstd = w.float(), rand((9,), "f32", 12).abs() + 0.5
    _, vals, meta, _ = sp.prune_compress(rand((64, 128), "bf16", 5))
    X, bias, res = rand((48, 128), "bf16", 6), rand((64,), "f32", 7), rand((48, 64), "bf16", 8)
    i8 = (rand((64, 128), "f32", 9) * 40).clamp(-127, 127).to(torch.int8)
    _, v8, m8, _ = sp.prune_compress(i8)
    X8 = (rand((32, 128), "f32", 10) * 40).clamp(-127, 127).to(torch.int8)
    rs, cs = rand((64,), "f32", 13), rand((32,), "f32", 14)
    wide = rand((9, 1040), "bf16", 11)
    yield lambda: sp.rms_norm(x, w)
    yield lambda: sp.rms_norm(x, w32, eps=1e-5, residual=r, quant="i8", with_rstd=True)
    yield lambda: sp.rms_norm(x, None, residual=r, quant="e5m2")
    yield lambda: sp.rms_norm(wide[:, 7:527], w, residual=wide[:, 520:], h_out=torch.empty_like(x), out=torch.empty_like(x))
    yield lambda: sp.rms_norm_backward(dy, x, w, rstd, dh=r)
    yield lambda: sp.rms_norm_backward(dy, x, None, rstd, out=torch.empty_like(x))
    yield lambda: sp.gated_act(wide[:, :520], wide[:, 520:], quant="e4m3")
    yield lambda: sp.gated_act(x, act="gelu_tanh")
    yield lambda: sp.gated_act_backward(dy, wide[:, :520], wide[:, 520:], act="gelu")
    yield lambda: sp.gated_act_backward(dy, x, act="relu")
    yield lambda: sp.act_backward(dy, x, act="silu", cd_col_major=True)
    yield lambda: sp.act_backward(dy, None, act=None, transposed=False)
    yield lambda: sp.linear(vals, meta, X, bias=bias, act="gelu", residual=res, pre=True, cd_col_major=True)
    yield lambda: sp.linear(vals, meta, X, cd="f32")
    yield lambda: sp.linear(v8, m8, X8, row_scale=rs, col_scale=cs)
    W = sp.decompress(vals, meta)
    dz, Xt = rand((48, 64), "bf16", 15), rand((128, 48), "bf16", 16)
    yield lambda: sp.linear_backward(dz, res, X, W, act="gelu", meta=meta, cd_col_major=True)
    yield lambda: sp.linear_backward(dz.T.contiguous(), None, Xt, W, b_row_major=True)
    yield lambda: sp.linear(i8, None, X8, a_is_dense=True, cd="f16", pre=torch.empty((64, 32), dtype=torch.float16, device="cuda"))


def test_native_and_python_forms_agree(sp, monkeypatch):
    native = [[None if v is None else v.clone() for v in flat(call())] for call in calls(sp)]
    monkeypatch.setattr(sp, "_native", Silent())
    for i, (call, want) in enumerate(zip(calls(sp), native)):
        got = flat(call())
        assert len(got) == len(want), i
        for a, b in zip(got, want):
            assert (a is None) == (b is None), i
            if a is not None:
                assert a.dtype == b.dtype and a.shape == b.shape and a.stride() == b.stride(), i
                assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)), i


def test_given_results_are_returned(sp):
    x = rand((5, 64), "f16", 1)
    out, h = torch.empty_like(x), torch.empty_like(x)
    y, h2, _, _ = sp.rms_norm(x, residual=x, h_out=h, out=out)
    assert y is out and h2 is h and sp.gated_act(x, x, out=out)[0] is out
    dg, du = sp.gated_act_backward(x, x, x, dg=out, du=h)
    assert dg is out and du is h and sp.act_backward(x, None, act=None)[0] is x


@pytest.mark.parametrize("silent", [False, True])
def test_refusals(sp, monkeypatch, silent):
    if silent:
        monkeypatch.setattr(sp, "_native", Silent())
    x, w, r = rand((4, 64), "bf16", 1), rand((64,), "bf16", 2), torch.rand(4, device="cuda")
    _, vals, meta, _ = sp.prune_compress(rand((64, 64), "bf16", 3))
    X = rand((32, 64), "bf16", 4)

    def refused(status, fn, *args, **kwargs):
        with pytest.raises(sp.Sp24Error) as e:
            fn(*args, **kwargs)
        assert e.value.status == status, (fn, e.value)
    refused(3, sp.rms_norm, x, w[:63])
    refused(2, sp.rms_norm, x, w.half())
    refused(3, sp.rms_norm, x, w, residual=x[:3])
    refused(2, sp.rms_norm, x, w, residual=x.half())
    refused(2, sp.rms_norm, x, w, quant="i4")
    refused(6, sp.rms_norm, x, w, eps=-1.0)
    refused(6, sp.rms_norm, x, w, h_out=x)
    refused(4, sp.rms_norm, rand((64, 4), "bf16", 5).T, w)
    refused(4, sp.rms_norm, x[:1].expand(4, 64), w)
    refused(6, sp.rms_norm, x, w.cpu())
    refused(2, sp.rms_norm, x, w, quant="i8", out=torch.empty_like(x))
    refused(3, sp.rms_norm_backward, x, x, w, r[:3])
    refused(2, sp.rms_norm_backward, x, x, w, r.half())
    refused(1, sp.rms_norm_backward, x, x, w, None)
    refused(3, sp.gated_act, x, x[:, :32])
    refused(6, sp.gated_act, x, x, act="tanh")
    refused(3, sp.gated_act_backward, x, x[:2], x)
    refused(6, sp.act_backward, x, x.cpu(), act="gelu")
    refused(1, sp.act_backward, x, None, act="gelu")
    refused(3, sp.linear, vals, meta, X[:, :32])
    refused(3, sp.linear, vals, meta[:100], X)
    refused(3, sp.linear, vals, meta, X, bias=torch.zeros(32, device="cuda"))
    refused(2, sp.linear, vals, meta, X, bias=torch.zeros(64, device="cuda", dtype=torch.bfloat16))
    refused(6, sp.linear, vals, meta, X, col_scale=torch.zeros(32, device="cuda"))
    refused(3, sp.linear, vals, meta, X, residual=X)
    refused(2, sp.linear, vals, meta, X.half())
    refused(2, sp.linear, vals, meta, X, cd="f16")
    refused(2, sp.linear, vals, meta, X, cd="f8")
    refused(1, sp.linear, vals, None, X)
    refused(6, sp.linear, vals, meta, X, act="swish")
    refused(3, sp.linear, vals, meta, X[:24])
    refused(3, sp.linear_backward, X, None, X, x)


@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 1), (3, 5), (8, 8)])
@pytest.mark.parametrize("K", [1, 7, 64, 250, 1531, 4096, 17000, 33001])
def test_outputs_stay_inside_their_rows(sp, offset, pad, K):
    """Results into the middle of wider matrices, at every alignment: what surrounds them keeps its bytes."""
    rows = 5
    x, u, w, dy = rand((rows, K), "bf16", 1, pad=pad), rand((rows, K), "bf16", 2), rand((K,), "bf16", 3), rand((rows, K), "bf16", 4)
    rstd = torch.rand(rows, device="cuda") + 0.5

    def room(dtype):
        full = torch.full((rows + 2, K + offset + pad + 3), 3, dtype=torch.int32, device="cuda").to(dtype)
        return full, full[1:rows + 1, offset:offset + K]

    def untouched(full):
        f = full.float()
        inside = torch.zeros_like(f, dtype=torch.bool)
        inside[1:rows + 1, offset:offset + K] = True
        return bool((f[~inside] == 3).all())
    def same(a, b, kind):
        """A row's sum is taken in another order where the row lies otherwise between boundaries: its factor may be a rounding or two
        off, and a result next to a border of its type one step (twice half a step)."""
        a, b = a.double(), b.double()
        step = torch.ones_like(a) if kind == "i8" else 2 * HALF_STEP[kind] * torch.maximum(a.abs(), b.abs()).clamp(min=TINY[kind])
        return bool(((a - b).abs() <= step).all())
    for quant, dtype in ((None, torch.bfloat16), ("i8", torch.int8), ("e4m3", torch.float8_e4m3fn)):
        (fy, y), (fh, h) = room(dtype), room(torch.bfloat16)
        want = sp.rms_norm(x, w, residual=u, quant=quant)
        sp.rms_norm(x, w, residual=u, quant=quant, h_out=h, out=y)
        assert untouched(fy) and untouched(fh) and torch.equal(h, want[1]) and same(y, want[0], quant or "bf16")
        fy, y = room(dtype)
        want = sp.gated_act(x, u, quant=quant)
        sp.gated_act(x, u, quant=quant, out=y)
        assert untouched(fy) and torch.equal(y.float(), want[0].float())
    (f1, o1), (f2, o2) = room(torch.bfloat16), room(torch.bfloat16)
    want = sp.gated_act_backward(dy, x, u)
    sp.gated_act_backward(dy, x, u, dg=o1, du=o2)
    assert untouched(f1) and untouched(f2) and torch.equal(o1, want[0]) and torch.equal(o2, want[1])
    (f1, o1), (f2, o2) = room(torch.bfloat16), room(torch.bfloat16)
    want = sp.rms_norm_backward(dy, x, w, rstd, dh=u)
    got = sp.rms_norm_backward(dy, x, w, rstd, dh=u, out=o1)
    assert untouched(f1) and same(o1, want[0], "bf16") and bool(((got[1] - want[1]).abs() <= 1e-5 * (1 + want[1].abs())).all())
    want = sp.act_backward(dy, x, act="gelu", transposed=False, bias=False)[0]
    sp.act_backward(dy, x, act="gelu", transposed=False, bias=False, out=o2)
    assert untouched(f2) and torch.equal(o2, want)
