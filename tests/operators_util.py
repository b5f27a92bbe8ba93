"""What the tests of the operators around the products share: inputs, plain implementations in 64 bits, tolerances."""
import math

import torch

DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32, "i8": torch.int8, "e4m3": torch.float8_e4m3fn,
         "e5m2": torch.float8_e5m2}
LARGEST = {"i8": 127.0, "e4m3": 448.0, "e5m2": 57344.0}
ACTS = [None, "relu", "gelu", "silu", "gelu_tanh"]
# A result is rounded once to its type: half a step of the value.
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24, "e4m3": 2.0 ** -4, "e5m2": 2.0 ** -3}
# The smallest normal value; below it the step is fixed.
TINY = {"f16": 2.0 ** -14, "bf16": 2.0 ** -126, "f32": 2.0 ** -126, "e4m3": 2.0 ** -6, "e5m2": 2.0 ** -14}


def rand(shape, dtype, seed, sigma=1.0, pad=0, device="cuda"):
    """N(0, sigma) of the type; with pad, a view whose rows are `pad` longer."""
    g = torch.Generator(device=device).manual_seed(seed)
    full = torch.randn((*shape[:-1], shape[-1] + pad), generator=g, device=device) * sigma
    return full.to(DTYPE[dtype])[..., :shape[-1]]


def close(got, want, dtype, arithmetic):
    """|got - want| is at most half a step of the type plus `arithmetic` (a bound on the FP32 arithmetic's error, per element), and what is not
    finite is so on both sides."""
    got, want = got.double(), want.double()
    finite = torch.isfinite(want)
    assert torch.equal(finite, torch.isfinite(got)), "finite in other places"
    assert torch.equal(torch.isnan(want), torch.isnan(got)), "NaN in other places"
    assert torch.equal(got[~finite & ~torch.isnan(want)], want[~finite & ~torch.isnan(want)])
    arithmetic = arithmetic if torch.is_tensor(arithmetic) else torch.as_tensor(arithmetic, dtype=torch.float64, device=got.device)
    bound = HALF_STEP[dtype] * (want.abs() + arithmetic).clamp(min=TINY[dtype]) + arithmetic
    over = ((got - want).abs() - bound).where(finite, torch.full_like(want, -1.0))
    assert over.numel() == 0 or float(over.max()) <= 0, f"over the bound by {float(over.max())} ({int((over > 0).sum())} of {over.numel()})"


def act64(z, act):
    """(act(z), act'(z)) in 64 bits."""
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * (1 - p)
    if act == "gelu":
        cdf = torch.special.ndtr(z)
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        p = torch.sigmoid(math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3))
        return z * p, p + z * p * (1 - p) * math.sqrt(8 / math.pi) * (1 + 3 * 0.044715 * z ** 2)
    return z, torch.ones_like(z)


def rms_norm64(h, weight, eps):
    """(norm of the rows of h, 1 / rms) in 64 bits."""
    h = h.double()
    rstd = 1 / torch.sqrt((h * h).mean(1) + eps)
    return h * rstd[:, None] * (1 if weight is None else weight.double()), rstd


def check_codes(codes, scale, n, kind, arithmetic):
    """8-bit codes and row scales of n (64 bits): scale = max |n| / L within 2^-21 (a handful of FP32 roundings: the row's factor, the product, 1 / L),
    codes the nearest ones of n / scale.  An element may be half a step of its code off, and by `arithmetic` (relative, of n / scale)."""
    L = LARGEST[kind]
    want = n.abs().amax(1) / L
    assert bool(((scale.double() - want).abs() <= 2.0 ** -21 * want).all())
    v = torch.where(want[:, None] > 0, n / want.clamp(min=1e-300)[:, None], torch.zeros_like(n))
    got = codes.double()
    if kind == "i8":
        bound = 0.5 + arithmetic * v.abs()
    else:
        bound = HALF_STEP[kind] * (v.abs() * (1 + arithmetic)).clamp(min=TINY[kind]) + arithmetic * v.abs()
    assert bool(((got - v).abs() <= bound).all()), float(((got - v).abs() - bound).max())
