"""GELU, its slope and 8-bit rows of it where the normal distribution's Phi is small: the bound is relative to the value, not to z."""
import pytest
import torch

from operators_util import DTYPE, HALF_STEP, LARGEST, TINY, close, rand

pytestmark = pytest.mark.gpu


def relative(z):
    """Share of Phi(z), z < 0, that FP32 arithmetic may lose, in units of 2^-24: t = 1 / (1 + 0.304 |z|) is off by 3 (its sum 1, the
    reciprocal 2), which passes to Phi exp(z^2 / 2) as at most 2.63 of itself (its logarithmic slope at z = 0 by t: 0.798 / 0.304); eight steps of
    the polynomial, of terms whose sum is at most 2.2 of the value, 3 each; the fit 1.4; the exponential 4; three products 3: 23 of 32.
    And z^2 / 2 log2(e), rounded three times (the constant half as much), makes the exponential off by z^2 / 2 times 2.5."""
    return 2.0 ** -19 + 1.25 * 2.0 ** -24 * z.double() ** 2


def gelu64(z):
    """(GELU, its slope, the sum of the slope's two terms' magnitudes) in 64 bits, Phi by erfc: (1 + erf) / 2, which torch.special.ndtr
    computes, has lost everything at -8.3."""
    z = z.double()
    cdf, density = torch.special.erfc(-z / 2 ** 0.5) / 2, torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
    return z * cdf, cdf + z * density, cdf + z.abs() * density


@pytest.fixture(scope="module")
def sp():
    from paper_2104_08378_b200 import binding
    return binding


def tail(lo, hi, shape, t="f32"):
    n = 1
    for s in shape:
        n *= s
    return -torch.linspace(lo, hi, n, dtype=torch.float64, device="cuda").reshape(shape).to(DTYPE[t])


@pytest.mark.parametrize("t", ["f16", "bf16", "f32"])
def test_values_and_slopes(sp, t):
    z = tail(0.25, 12.5, (8, 1024), t)
    u, dy = rand(z.shape, t, 1), rand(z.shape, t, 2)
    value, slope, terms = gelu64(z)
    close(sp.gated_act(z, act="gelu")[0], value, t, relative(z) * value.abs())
    close(sp.gated_act(z, u, act="gelu")[0], value * u.double(), t, relative(z) * (value * u.double()).abs())
    dg, du = sp.gated_act_backward(dy, z, u, act="gelu")
    f = dy.double() * u.double()
    close(dg, f * slope, t, relative(z) * terms * f.abs())
    close(du, dy.double() * value, t, relative(z) * (dy.double() * value).abs())
    dz, _, _ = sp.act_backward(dy, z, act="gelu", cd_col_major=True)
    close(dz, dy.double() * slope, t, relative(z) * terms * dy.double().abs())


@pytest.mark.parametrize("quant", ["i8", "e4m3", "e5m2"])
def test_eight_bit_rows_in_the_tail(sp, quant):
    z, u = tail(4.5, 6.0, (16, 520)), rand((16, 520), "f32", 3)
    codes, scale = sp.gated_act(z, u, act="gelu", quant=quant)
    n = gelu64(z)[0] * u.double()
    want = n.abs().amax(1) / LARGEST[quant]
    most = relative(z).max() + 2.0 ** -21                 # (a handful of roundings of the scale and of the codes' factor)
    assert bool(((scale.double() - want).abs() <= most * want).all())
    v = n / want[:, None]
    off = 2 * most * v.abs()                              # the value's error and the scale's
    bound = (0.5 if quant == "i8" else HALF_STEP[quant] * (v.abs() + off).clamp(min=TINY[quant])) + off
    assert bool(((codes.double() - v).abs() <= bound).all())


@pytest.mark.parametrize("ab,cd", [("bf16", "f32"), ("bf16", "bf16"), ("i8", "f32"), ("i8", "f16"), ("e4m3", "f32"), ("f32", "f32")])
def test_epilogue(sp, ab, cd):
    """Tokens of zeros: the bias alone is what GELU is applied to."""
    if ab == "i8":
        W, X = torch.ones((512, 128), dtype=torch.int8, device="cuda"), torch.zeros((64, 128), dtype=torch.int8, device="cuda")
    else:
        W, X = rand((512, 128), ab, 4), torch.zeros((64, 128), device="cuda").to(DTYPE[ab])
    _, vals, meta, _ = sp.prune_compress(W)
    z = tail(0.25, 12.5, (512,))
    value = gelu64(z)[0]
    for cols in (False, True):
        y = sp.linear(vals, meta, X, bias=z, act="gelu", cd=cd, cd_col_major=cols)
        y = y if cols else y.T
        close(y, value.expand_as(y), cd, relative(z) * value.abs())
