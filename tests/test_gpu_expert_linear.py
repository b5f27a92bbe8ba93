"""Products of every expert's rows with its own weights, and their gradients, against plain implementations in 64 bits."""
import math

import pytest
import torch

from operators_util import ACTS, DTYPE, act64, close, rand

pytestmark = pytest.mark.gpu


# As for the linear layer: FP32 accumulation in chains of K / 32 + 32 additions that truncate, then the epilogue's roundings.
def z_error(K, scale, z):
    return (K / 32 + 34) * 2.0 ** -23 * scale + 2.0 ** -22 * z.abs()


def d_error(K, scale, z, d):
    return 1.13 * z_error(K, scale, z) + 2.0 ** -20 * z.abs() + 2.0 ** -23 * d.abs()


@pytest.fixture(scope="module")
def sp():
    from paper_2104_08378_b200 import binding
    return binding


def operand(shape, ab, seed):
    if ab == "i8":
        g = torch.Generator(device="cuda").manual_seed(seed)
        return torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8)
    return rand(shape, ab, seed)


def weights(sp, E, M, K, ab, dense, seed):
    """(W as multiplied [E, M, K], A operand, meta)."""
    W = operand((E, M, K), ab, seed)
    if dense:
        return W, W, None
    W = torch.stack([sp.prune(W[e]) for e in range(E)]) if W.element_size() == 2 else torch.stack(
        [sp.prune_compress(W[e])[0] for e in range(E)])
    return (W,) + sp.expert_compress(W)


def check(sp, counts, M, K, ab, cd, act, seed, *, dense=False, bias=True, residual=True, scales=True, pre=True, pad=0, before=0, behind=3):
    E, ends = len(counts), [before]
    for n in counts:
        ends.append(ends[-1] + n)
    rows = ends[-1] + behind
    W, A, meta = weights(sp, E, M, K, ab, dense, seed)
    X = operand((rows, K), ab, seed + 1)
    one_byte = ab in ("i8", "e4m3", "e5m2")
    norm = math.sqrt(K) * (5400.0 if ab == "i8" else 1.0)
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    row_scale = (torch.rand((E, M), generator=g, device="cuda") + 0.5) / norm if scales else None
    col_scale = torch.rand(rows, generator=g, device="cuda") + 0.5 if scales and one_byte else None
    b = rand((E, M), "f32", seed + 3) if bias else None
    r = rand((rows, M), cd, seed + 4, pad=pad) if residual else None
    out = torch.full((rows, M + pad), 7.0, device="cuda").to(DTYPE[cd])
    kept = torch.full((rows, M), 5.0, device="cuda").to(DTYPE[cd]) if pre else None
    got = sp.expert_linear(A, meta, X, torch.tensor(ends, dtype=torch.int32, device="cuda"), bias=b, act=act, residual=r, row_scale=row_scale,
                           col_scale=col_scale, pre=kept if pre else False, out=out[:, :M], cd=cd, a_is_dense=dense)
    assert sp.gemm_status() == 0
    if pre:
        assert got[1] is kept
    for e in range(E):
        lo, hi = ends[e], ends[e + 1]
        x, w = X[lo:hi].double(), W[e].double()
        f = torch.ones((hi - lo, M), dtype=torch.float64, device="cuda")
        if row_scale is not None:
            f = f * row_scale[e].double()
        if col_scale is not None:
            f = f * col_scale[lo:hi, None].double()
        z, scale = x @ w.T * f, x.abs() @ w.abs().T * f.abs()
        z = z if b is None else z + b[e].double()
        d = act64(z, act)[0] + (0 if r is None else r[lo:hi].double())
        if pre:
            close(kept[lo:hi], z, cd, z_error(K, scale, z))
        close(out[lo:hi, :M], d, cd, d_error(K, scale, z, d))
    # what belongs to no expert, and what lies beside the rows, is as it was
    assert bool((out[:ends[0]] == 7).all()) and bool((out[ends[-1]:] == 7).all()) and bool((out[:, M:] == 7).all())
    if pre:
        assert bool((kept[:ends[0]] == 5).all()) and bool((kept[ends[-1]:] == 5).all())


TYPES = [("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("i8", "bf16"), ("i8", "f16"), ("i8", "f32"), ("e4m3", "bf16"), ("e4m3", "f16"),
         ("e5m2", "f32"), ("e5m2", "bf16")]


@pytest.mark.parametrize("ab,cd", TYPES)
@pytest.mark.parametrize("act", ACTS)
def test_types_and_activations(sp, ab, cd, act):
    check(sp, [5, 0, 33, 1], 160, 416, ab, cd, act, 1)
    check(sp, [200, 31, 0, 260], 288, 224, ab, cd, act, 2, residual=False, pre=False)


@pytest.mark.parametrize("ab,cd", [("bf16", "bf16"), ("f16", "f32"), ("i8", "bf16"), ("e4m3", "f16")])
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("counts,M,K", [([1], 32, 32), ([0, 0, 1, 0], 128, 4096), ([2] * 64, 96, 256), ([300], 4096, 64), ([17, 130, 64, 1, 0, 250], 1184, 1024),
                                        ([0] * 30 + [129] + [0] * 33, 544, 544), ([700, 225, 1], 256, 2080), ([40, 224, 448, 449], 800, 96),
                                        ([1] * 1000 + [0] * 24, 32, 64), ([3000, 2, 1100], 2080, 160)])
def test_sizes(sp, ab, cd, dense, counts, M, K):
    check(sp, counts, M, K, ab, cd, "gelu", 1, dense=dense, before=5)
    check(sp, counts, M, K, ab, cd, None, 2, dense=dense, bias=False, residual=False, scales=False, pre=False, behind=0)
    check(sp, counts, M, K, ab, cd, "silu", 3, dense=dense, pad=16, pre=False)


@pytest.mark.parametrize("tile", ["1x32x1", "1x64x1", "1x96x1", "1x128x1", "2x64x1", "2x96x1", "2x128x1", "2x160x1", "2x192x1", "2x224x1"])
@pytest.mark.parametrize("ab,cd", [("bf16", "f32"), ("f16", "f16"), ("i8", "bf16"), ("e4m3", "f16")])
def test_every_width(sp, force_tile, tile, ab, cd):
    """Whatever tile a problem is given: experts that end inside one, at its edge, and with a row more."""
    n = int(tile.split("x")[1])
    force_tile(tile)
    check(sp, [n - 1, n, 1, 0, n + 1, 2 * n + 17], 288, 544, ab, cd, "gelu", 1)
    check(sp, [3, 2 * n], 160, 96, ab, cd, None, 2, bias=False, residual=False, pre=False)


@pytest.mark.parametrize("ab", ["bf16", "i8"])
def test_every_dense_width(sp, force_tile, ab):
    for tile in ("1x64x1", "1x128x1", "2x64x1", "2x128x1", "2x160x1", "2x224x1", "2x256x1"):
        force_tile(tile)
        check(sp, [255, 0, 256, 1, 257], 288, 416, ab, "bf16", "silu", 1, dense=True)


@pytest.mark.parametrize("tile", ["1x32x1", "1x128x1", "2x64x1", "2x96x1", "2x160x1", "2x192x1", "2x256x1"])
def test_every_width_of_the_gradient(sp, force_tile, tile):
    force_tile(tile)
    check_gradients(sp, [64, 0, 96, 16, 272], 160, 304, "bf16", "silu", 1)


def test_the_residual_may_be_the_result(sp):
    W, A, meta = weights(sp, 3, 64, 128, "bf16", False, 1)
    X, r = rand((50, 128), "bf16", 2), rand((50, 64), "bf16", 3)
    offsets = torch.tensor([0, 20, 20, 50], dtype=torch.int32, device="cuda")
    want = sp.expert_linear(A, meta, X, offsets, residual=r)
    assert sp.expert_linear(A, meta, X, offsets, residual=r, out=r) is r and torch.equal(r, want)


def test_one_expert_is_the_linear_layer(sp):
    """The same kernel's arithmetic: K in the same order whatever the tile, so the same bits."""
    for ab in ("bf16", "i8"):
        W, A, meta = weights(sp, 1, 256, 512, ab, False, 1)
        X = operand((96, 512), ab, 2)
        got = sp.expert_linear(A, meta, X, torch.tensor([0, 96], dtype=torch.int32, device="cuda"))
        assert torch.equal(got, sp.linear(A[0], meta[0], X, cd_col_major=True))


def test_offsets_out_of_range_or_order(sp):
    """Offsets that expert_order does not give: those outside count as the nearest that are not, and no row outside is touched."""
    W, A, meta = weights(sp, 4, 64, 64, "f16", False, 1)
    X = rand((40, 64), "f16", 2)
    whole = torch.full((60, 64), 7.0, dtype=torch.float16, device="cuda")
    out = whole[10:50]
    for given, meant in (([-5, 10, 20, 30, 99], [0, 10, 20, 30, 40]), ([0, 30, 20, 35, 40], [0, 30, 30, 35, 40]), ([50, 0, 0, 0, 0], [40] * 5),
                         ([0, 0, 0, 0, -1], [0] * 5)):
        whole.fill_(7.0)
        sp.expert_linear(A, meta, X, torch.tensor(given, dtype=torch.int32, device="cuda"), out=out)
        got = whole.clone()
        whole.fill_(7.0)
        sp.expert_linear(A, meta, X, torch.tensor(meant, dtype=torch.int32, device="cuda"), out=out)
        assert torch.equal(got, whole) and bool((got[:10] == 7).all()) and bool((got[50:] == 7).all())


def test_no_rows(sp):
    W, A, meta = weights(sp, 2, 64, 64, "bf16", False, 1)
    assert sp.expert_linear(A, meta, torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")).shape == (0, 64)
    check(sp, [0, 0], 64, 64, "bf16", "bf16", "relu", 1)


# dz is rounded once (half a step) before the products, which accumulate in FP32 as above; the slope is off by at most 2^-19.
def check_gradients(sp, counts, M, K, t, act, seed, *, masked=True, pad=0, behind=16):
    E, ends = len(counts), [0]
    for n in counts:
        ends.append(ends[-1] + n)
    rows = ends[-1] + behind
    W, A, meta = weights(sp, E, M, K, t, False, seed)
    X, dy, pre = rand((rows, K), t, seed + 1), rand((rows, M), t, seed + 2, pad=pad), rand((rows, M), t, seed + 3, pad=pad)
    X[ends[-1]:], dy[ends[-1]:] = float("nan"), float("nan")       # what belongs to no expert reaches no gradient
    dX, dW, db = sp.expert_linear_backward(dy, pre if act else None, X, W, torch.tensor(ends, dtype=torch.int32, device="cuda"), act=act,
                                           meta=meta if masked else None)
    assert sp.gemm_status() == 0
    half = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}[t]
    for e in range(E):
        lo, hi = ends[e], ends[e + 1]
        x, w = X[lo:hi].double(), W[e].double()
        dz = dy[lo:hi].double() * act64(pre[lo:hi].double(), act)[1]
        size = dy[lo:hi].double().abs() * 1.13
        off = (half if act else 0.0) * dz.abs() + (2.0 ** -18 * size if act else 0.0)   # of dz as the products have it
        if hi > lo:
            close(dX[lo:hi], dz @ w, t, off @ w.abs() + z_error(M, dz.abs() @ w.abs(), dz @ w))
        want, err = dz.T @ x, off.T @ x.abs() + z_error(max(16, hi - lo), dz.abs().T @ x.abs(), dz.T @ x)
        if masked:
            want, err = want * (w != 0), err * (w != 0)
        close(dW[e], want, t, err)
        close(db[e], dz.sum(0), "f32", (hi - lo + 8) * 2.0 ** -24 * dz.abs().sum(0) + (2.0 ** -18 * size.sum(0) if act else 0.0))


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("act", ACTS)
def test_gradients(sp, t, act):
    check_gradients(sp, [16, 0, 48, 160], 96, 160, t, act, 1)
    check_gradients(sp, [320, 16, 0, 272], 288, 224, t, act, 2, pad=3)


@pytest.mark.parametrize("counts,M,K", [([16], 16, 16), ([0, 0, 16], 128, 4096), ([2048], 64, 48), ([16] * 64, 48, 272), ([144, 1008, 0, 32], 1184, 736),
                                        ([0, 0], 32, 64), ([640, 656, 16], 2048, 144), ([16] * 1000 + [0] * 24, 16, 32)])
def test_gradients_of_sizes(sp, counts, M, K):
    check_gradients(sp, counts, M, K, "bf16", "gelu", 1, masked=False)
    check_gradients(sp, counts, M, K, "f16", None, 2, behind=0)


def test_weights_gradient_of_experts_that_are_not_placed_at_16(sp):
    """NaN instead of a sum over other experts' rows; the others' gradients, and those of the rows, are as ever."""
    W, A, meta = weights(sp, 3, 64, 64, "bf16", False, 1)
    X, dy = rand((64, 64), "bf16", 2), rand((64, 64), "bf16", 3)
    good = sp.expert_linear_backward(dy, None, X, W, torch.tensor([0, 16, 32, 64], dtype=torch.int32, device="cuda"))
    dX, dW, db = sp.expert_linear_backward(dy, None, X, W, torch.tensor([0, 16, 27, 64], dtype=torch.int32, device="cuda"))
    assert torch.equal(dW[0], good[1][0]) and bool(dW[1].isnan().all()) and bool(dW[2].isnan().all())
    assert torch.equal(dX[:27], good[0][:27]) and not bool(dX.isnan().any()) and not bool(db.isnan().any())


def test_gradients_against_differences(sp):
    """sum of dD * D changes by what the gradients say, in 64 bits around the inputs."""
    W, A, meta = weights(sp, 2, 32, 64, "f16", False, 1)
    X, dy = rand((48, 64), "f16", 2), rand((48, 32), "f16", 3)
    ends = [0, 16, 48]
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    _, pre = sp.expert_linear(A, meta, X, offsets, act="silu", pre=True)
    dX, dW, _ = sp.expert_linear_backward(dy, pre, X, W, offsets, act="silu", meta=meta)
    step_x, step_w = rand((48, 64), "f32", 4).double(), rand((2, 32, 64), "f32", 5).double() * (W != 0)

    def f(h):
        return sum((act64((X[lo:hi].double() + h * step_x[lo:hi]) @ (W[e].double() + h * step_w[e]).T, "silu")[0] * dy[lo:hi].double()).sum()
                   for e, (lo, hi) in enumerate(zip(ends, ends[1:])))
    h = 1e-5
    slope = (f(h) - f(-h)) / (2 * h)
    got = (dX.double() * step_x).sum() + (dW.double() * step_w).sum()
    # every product of a step and a gradient is off by two half steps (dz and the result) and z's rounding (2^-11 |z| times a slope's slope of at most 0.5)
    size = (dX.double() * step_x).abs().sum() + (dW.double() * step_w).abs().sum() + (dy.double().abs() @ (W.double().abs().sum(0))).sum()
    assert abs(float(got - slope)) <= 4 * 2.0 ** -11 * float(size)
