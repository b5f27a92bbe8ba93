"""The gated activation, its gradient and the activation's gradient in both orders, against plain implementations in 64 bits."""
import pytest
import torch

from operators_util import ACTS, DTYPE, act64, check_codes, close, rand

pytestmark = pytest.mark.gpu
# FP32 arithmetic of an activation: Phi by a polynomial with an absolute error of 3e-7 (the published bound 0.75e-7 and its
# roundings) < 2^-21, the logistic and its exponential to 2^-20 of their value for |z| < 16, a few products.  So an
# activation is off by at most 2^-20 max(|z|, |act(z)|), a slope by 2^-18 (its terms are up to 1.2, the tanh form's inner
# derivative up to 2 sqrt(2/pi) (1 + 0.134 z^2) where it is not switched off, below 8 there).
VALUE, SLOPE = 2.0 ** -20, 2.0 ** -17


@pytest.fixture(scope="module")
def sp():
    from paper_2104_08378_b200 import binding
    return binding


SHAPES = [(1, 1), (3, 7), (5, 64), (9, 255), (33, 1000), (2, 4096), (3, 8191), (2, 12288), (1, 40000)]


@pytest.mark.parametrize("t", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
def test_values(sp, t, act):
    for rows, F in SHAPES:
        for gated, pad in ((True, 0), (True, 5), (False, 3)):
            gu = rand((rows, 2 * F), t, 1, sigma=2.0, pad=pad)
            g, u = gu[:, :F], gu[:, F:] if gated else None
            y, scale = sp.gated_act(g, u, act=act)
            a, f = act64(g.double(), act)[0], (1.0 if u is None else u.double())
            assert scale is None
            close(y, a * f, t, VALUE * g.double().abs() * (1.0 if u is None else u.double().abs()))


@pytest.mark.parametrize("quant", ["i8", "e4m3", "e5m2"])
@pytest.mark.parametrize("t", ["f16", "bf16", "f32"])
def test_eight_bit_results(sp, t, quant):
    for act in (None, "silu", "gelu"):
        for rows, F in SHAPES:
            g, u = rand((rows, F), t, 2, pad=3), rand((rows, F), t, 3)
            u[rows // 2] = 0
            y, scale = sp.gated_act(g, u, act=act, quant=quant)
            n = act64(g.double(), act)[0] * u.double()
            assert y.dtype == DTYPE[quant] and float(scale[rows // 2]) == 0 and not y[rows // 2].double().any()
            # (in the far tail of an activation the error counts against z, not against the small value: |n| there is below 2^-3 of
            # the row's steps anyway, so an absolute share of the code's step covers it)
            L = {"i8": 127.0, "e4m3": 448.0, "e5m2": 57344.0}[quant]
            want = n.abs().amax(1) / L
            err = VALUE * (g.double() * u.double()).abs()
            assert bool(((scale.double() - want).abs() <= 2.0 ** -21 * want + err.amax(1) / L).all())
            s = scale.double().clamp(min=1e-300)[:, None]
            step = 0.5 if quant == "i8" else None
            v = torch.where(want[:, None] > 0, n / s, torch.zeros_like(n))
            half = {"e4m3": 2.0 ** -4, "e5m2": 2.0 ** -3}
            slack = 2.0 ** -20 * v.abs() + torch.where(want[:, None] > 0, err / s, torch.zeros_like(err))
            bound = step + slack if step else half[quant] * (v.abs() + slack).clamp(min=2.0 ** -6 if quant == "e4m3" else 2.0 ** -14) + slack
            assert bool(((y.double() - v).abs() <= bound).all())
    x = rand((4, 300), t, 4)                                    # rows themselves, quantised
    y, scale = sp.gated_act(x, act=None, quant=quant)
    check_codes(y, scale, x.double(), quant, 2.0 ** -20)


@pytest.mark.parametrize("quant", ["i8", "e4m3", "e5m2"])
def test_rows_that_are_not_finite(sp, quant):
    g, u = rand((4, 260), "bf16", 5), rand((4, 260), "bf16", 6)
    clean, clean_scale = sp.gated_act(g, u, quant=quant)
    g[1, 3], u[2, 259] = float("nan"), float("inf")
    y, scale = sp.gated_act(g, u, quant=quant)
    for row in (0, 3):
        assert torch.equal(y[row].view(torch.uint8), clean[row].view(torch.uint8)) and scale[row] == clean_scale[row]
    assert torch.isnan(scale[1:3]).all()
    assert not y[1:3].float().any() if quant == "i8" else torch.isnan(y[1:3].float()).all()


@pytest.mark.parametrize("act", ACTS)
def test_far_arguments(sp, act):
    """Activations and slopes where their exponentials have long left the range."""
    z = torch.tensor([[0.0, -0.0, 30.0, -30.0, 100.0, -100.0, 1e4, -1e4, 1e20, -1e20, 3e38, -3e38]], device="cuda")
    value, slope = act64(z.double(), act)
    one = torch.ones_like(z)
    # exp(-z) = 2^(-z log2 e) with the product rounded: an exponent that is off by |z| log2(e) 2^-24 makes the power off by
    # |z| 2^-24 of its value, 2^-19.1 at 30; beyond about 88 the value is below the smallest float.
    close(sp.gated_act(z, act=act)[0], value, "f32", (VALUE + z.double().abs().clamp(max=128) * 2.0 ** -24) * value.abs() + 1e-30)
    close(sp.gated_act_backward(one, z, act=act)[0], slope.nan_to_num(1.0), "f32", SLOPE)


@pytest.mark.parametrize("t", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
def test_gradient(sp, t, act):
    for rows, F in SHAPES:
        for gated, pad in ((True, 0), (True, 5), (False, 3)):
            gu, dy = rand((rows, 2 * F), t, 7, sigma=2.0, pad=pad), rand((rows, F), t, 8)
            g, u = gu[:, :F], gu[:, F:] if gated else None
            dg, du = sp.gated_act_backward(dy, g, u, act=act)
            value, slope = act64(g.double(), act)
            f = dy.double() * (1.0 if u is None else u.double())
            close(dg, f * slope, t, SLOPE * f.abs())
            assert (du is None) == (u is None)
            if u is not None:
                close(du, dy.double() * value, t, VALUE * (dy.double() * g.double()).abs())
                both = torch.empty_like(gu)                     # into the halves of one matrix
                sp.gated_act_backward(dy, g, u, act=act, dg=both[:, :F], du=both[:, F:])
                assert torch.equal(both, torch.cat((dg, du), 1))


@pytest.mark.parametrize("act", ACTS[1:])
def test_gradient_against_differences(sp, act):
    g = torch.linspace(-4.03, 4.05, 96, device="cuda").reshape(3, 32).double()
    u, dy = rand((3, 32), "f32", 9).double(), rand((3, 32), "f32", 10).double()
    dg, du = sp.gated_act_backward(dy.float(), g.float(), u.float(), act=act)
    step = 1e-4
    slope = (act64(g + step, act)[0] - act64(g - step, act)[0]) / (2 * step)
    # (differences: step^2 / 6 times a third derivative below 3; FP32 inputs and arithmetic: 2^-17 of the terms)
    assert float((dg.double() - dy * u * slope).abs().max()) <= 1e-7 + SLOPE * float((dy * u).abs().max())
    assert float((du.double() - dy * act64(g, act)[0]).abs().max()) <= 1e-7 + SLOPE * float((dy * g).abs().max())


@pytest.mark.parametrize("t", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("tokens_out", [True, False])
def test_act_backward(sp, t, act, tokens_out):
    for rows, cols in [(1, 1), (1, 300), (300, 1), (64, 64), (65, 130), (16, 4096), (1000, 272), (333, 1001)]:
        dy, z = rand((rows, cols), t, 11, pad=3), rand((rows, cols), t, 12, sigma=2.0)
        dz, dzt, db = sp.act_backward(dy, z, act=act, cd_col_major=tokens_out)
        want = dy.double() * act64(z.double(), act)[1]
        close(dz, want, t, SLOPE * dy.double().abs())
        assert (dz is dy) == (act is None) and torch.equal(dzt, dz.T)
        axis = 0 if tokens_out else 1
        close(db, want.sum(axis), "f32", (SLOPE + 2.0 ** -17) * dy.double().abs().sum(axis))
        again = sp.act_backward(dy, z, act=act, cd_col_major=tokens_out)
        assert torch.equal(again[2], db)
        only, none, no_bias = sp.act_backward(dy, z, act=act, transposed=False, bias=False)
        assert none is None and no_bias is None and torch.equal(only, dz)
        if act is not None:
            a = z.clone()
            assert torch.equal(sp.act_backward(dy, a, act=act, out=a)[0], dz)


def test_no_rows_and_in_place(sp):
    e = rand((0, 64), "bf16", 1)
    y, scale = sp.gated_act(e, e, quant="i8")
    assert y.shape == (0, 64) and scale.shape == (0,) and sp.gated_act_backward(e, e, e)[1].shape == (0, 64)
    dz, dzt, db = sp.act_backward(e, e, act="gelu", cd_col_major=True)
    assert dzt.shape == (64, 0) and not db.any() and db.shape == (64,)
    g, u = rand((7, 520), "f16", 13), rand((7, 520), "f16", 14)
    y, _ = sp.gated_act(g, u)
    a = g.clone()
    assert torch.equal(sp.gated_act(a, u, out=a)[0], y)
    dy = rand((7, 520), "f16", 15)
    dg, du = sp.gated_act_backward(dy, g, u)
    a, b = g.clone(), u.clone()
    sp.gated_act_backward(dy, a, b, dg=b, du=a)                 # each in place of the other's input
    assert torch.equal(b, dg) and torch.equal(a, du)


def test_captured(sp):
    gu, dy = rand((48, 2080), "bf16", 16), rand((48, 1040), "bf16", 17)

    def step():
        y, scale = sp.gated_act(gu[:, :1040], gu[:, 1040:], quant="e4m3")
        return (y, scale) + sp.gated_act_backward(dy, gu[:, :1040], gu[:, 1040:]) + sp.act_backward(dy, gu[:, :1040], act="gelu")
    want = [v.clone() for v in step()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))


@pytest.mark.parametrize("t,F", [("bf16", 12288), ("bf16", 9001), ("f16", 8192), ("f32", 4096), ("f32", 5000), ("bf16", 5120), ("bf16", 20000)])
def test_a_row_does_not_depend_on_the_others(sp, t, F):
    """Enough rows for every arrangement of teams: the same bits as a few by themselves."""
    rows = 4800
    g, u = rand((rows, F), t, 18), rand((rows, F), t, 19)
    for quant in (None, "i8"):
        y, scale = sp.gated_act(g, u, act="gelu", quant=quant)
        for some in (slice(0, 1), slice(3201, 3209), slice(4400, 4800)):
            y2, scale2 = sp.gated_act(g[some], u[some], act="gelu", quant=quant)
            assert torch.equal(y2, y[some]) and (quant is None or torch.equal(scale2, scale[some]))


def test_offsets_past_32_bits(sp):
    """Rows 2^31 + 8 elements apart, of operands and results."""
    ld = 2 ** 31 + 8
    room = [torch.empty(ld + 64, dtype=torch.bfloat16, device="cuda").as_strided((2, 64), (ld, 1)) for _ in range(3)]
    g, u, y = room
    g.copy_(rand((2, 64), "bf16", 20))
    u.copy_(rand((2, 64), "bf16", 21))
    a, slope = act64(g.double(), "silu")
    sp.gated_act(g, u, out=y)
    close(y, a * u.double(), "bf16", VALUE * (g.double() * u.double()).abs())
    dg, du = sp.gated_act_backward(y, g, u)
    close(dg, y.double() * u.double() * slope, "bf16", SLOPE * (y.double() * u.double()).abs())
    dz, dzt, db = sp.act_backward(u, g, act="silu", cd_col_major=True, out=y)
    close(dz, u.double() * slope, "bf16", SLOPE * u.double().abs())
    assert torch.equal(dzt, dz.T)
