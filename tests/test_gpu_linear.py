"""The linear layer's product with scales, bias, activation and residual, and its gradients, against plain implementations in 64
bits; and the operators of a feed-forward layer one after the other."""
import math
import os
import subprocess
import sys

import pytest
import torch

from operators_util import ACTS, DTYPE, act64, close, rand, rms_norm64

pytestmark = pytest.mark.gpu
# FP32 accumulation of K products, exact each (TF32: of inputs that the mode takes exactly): at most K additions, of which the
# tensor cores truncate (2^-23 each) sums of no more than (|A| . |B|)_ij.  The instructions add 32 or more products at a time, so K / 32 + 32 of them
# bound a chain.  Epilogue: two roundings of the scales, one multiply-add, the activation (2^-20 of |z|; slopes of activations are at most 1.13, so an error of
# z passes on as 1.13 of itself), the residual's addition.
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
    x = rand(shape, ab, seed)
    return (x.view(torch.int32) & -8192).view(torch.float32) if ab == "f32" else x    # TF32: 13 mantissa bits less


def layer(sp, M, N, K, ab, dense, b_rows, seed):
    """(W as multiplied, A operand, meta, X)."""
    W = operand((M, K), ab, seed)
    X = operand((K, N) if b_rows else (N, K), ab, seed + 1)
    if dense:
        return W, W, None, X
    W, vals, meta, _ = sp.prune_compress(W)
    return W, vals, meta, X


def reference(W, X, b_rows, row_scale, col_scale, bias):
    """(z, what its accumulation's error scales with) in 64 bits, M x N."""
    W, X = W.double(), X.double() if b_rows else X.double().T
    f = torch.ones(W.shape[0], X.shape[1], dtype=torch.float64, device="cuda")
    if row_scale is not None:
        f = f * row_scale.double()[:, None]
    if col_scale is not None:
        f = f * col_scale.double()[None]
    z = W @ X * f
    return z if bias is None else z + bias.double()[:, None], W.abs() @ X.abs() * f.abs()


def check(sp, M, N, K, ab, cd, act, seed, *, dense=False, b_rows=False, cols=False, bias=True, residual=True, scales=True, pre=True, pad=0):
    W, A, meta, X = layer(sp, M, N, K, ab, dense, b_rows, seed)
    one_byte = ab in ("i8", "e4m3", "e5m2")
    norm = math.sqrt(K) * (5400.0 if ab == "i8" else 1.0)
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    row_scale = (torch.rand(M, generator=g, device="cuda") + 0.5) / norm if scales else None
    col_scale = torch.rand(N, generator=g, device="cuda") + 0.5 if scales and one_byte else None
    b = rand((M,), "f32", seed + 3) if bias else None
    shape = (N, M) if cols else (M, N)
    r = rand(shape, cd, seed + 4, pad=pad) if residual else None
    out = torch.empty((shape[0], shape[1] + pad), dtype=DTYPE[cd], device="cuda")[:, :shape[1]] if pad else None
    got = sp.linear(A, meta, X, bias=b, act=act, residual=r, row_scale=row_scale, col_scale=col_scale, pre=pre, out=out, cd=cd,
                    a_is_dense=dense, b_row_major=b_rows, cd_col_major=cols)
    assert sp.gemm_status() == 0
    z, scale = reference(W, X, b_rows, row_scale, col_scale, b)
    z, scale = (z.T, scale.T) if cols else (z, scale)
    d = act64(z, act)[0] + (0 if r is None else r.double())
    if pre:
        got, got_z = got
        close(got_z, z, cd, z_error(K, scale, z))
    assert got.dtype == DTYPE[cd] and (out is None or got is out)
    close(got, d, cd, d_error(K, scale, z, d))


TYPES = [("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("i8", "bf16"), ("i8", "f16"), ("i8", "f32"),
         ("e4m3", "bf16"), ("e4m3", "f16"), ("e4m3", "f32"), ("e5m2", "bf16"), ("f32", "f32")]


@pytest.mark.parametrize("ab,cd", TYPES)
@pytest.mark.parametrize("act", ACTS)
def test_types_and_activations(sp, ab, cd, act):
    for i, (cols, residual) in enumerate([(False, False), (False, True), (True, False), (True, True)]):
        check(sp, 288, 224, 416, ab, cd, act, 10 * i, cols=cols, residual=residual)


@pytest.mark.parametrize("ab,cd", [("bf16", "bf16"), ("f16", "f32"), ("i8", "bf16"), ("e4m3", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("M,N,K", [(32, 32, 32), (128, 32, 4096), (160, 96, 12288), (4096, 32, 1024), (20000, 64, 256), (512, 1056, 544),
                                   (2080, 992, 768), (1184, 736, 1024)])
def test_sizes(sp, ab, cd, M, N, K):
    check(sp, M, N, K, ab, cd, "gelu", 1, cols=True)
    check(sp, M, N, K, ab, cd, "silu", 2, cols=False, bias=False, pad=16)
    check(sp, M, N, K, ab, cd, None, 3, cols=True, residual=False, scales=False, pre=False)


@pytest.mark.parametrize("ab,cd", [("bf16", "bf16"), ("f16", "f32"), ("i8", "f16"), ("e5m2", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("dense,b_rows", [(True, False), (False, True), (True, True)])
def test_dense_weights_and_the_other_order(sp, ab, cd, dense, b_rows):
    check(sp, 320, 288, 512, ab, cd, "gelu_tanh", 4, dense=dense, b_rows=b_rows, cols=True)
    check(sp, 1056, 480, 256, ab, cd, "relu", 5, dense=dense, b_rows=b_rows, cols=False)


@pytest.mark.parametrize("ab,cd", [("bf16", "bf16"), ("bf16", "f32"), ("i8", "bf16"), ("e4m3", "f16")])
@pytest.mark.parametrize("tile", ["1x128x1", "2x224x1", "2x224x2", "2x256x1", "2x240x1", "2x192x2", "1x128x2", "1x128x3"])
def test_every_tile_shape(sp, force_tile, ab, cd, tile):
    if (tile == "2x240x1" and (ab, cd) != ("bf16", "bf16")) or (tile == "2x192x2" and ab == "e4m3"):
        pytest.skip("not built")
    force_tile(tile)
    N = 96 if tile in ("1x128x2", "1x128x3") else 704
    for cols in (False, True):
        check(sp, 1120, N, 512, ab, cd, "silu", 6, cols=cols)
        check(sp, 1120, N, 512, ab, cd, "gelu", 7, cols=cols, residual=False, pre=False)


def test_the_residual_may_be_the_result(sp):
    for cols in (False, True):
        _, A, meta, X = layer(sp, 512, 320, 256, "bf16", False, False, 8)
        r = rand((320, 512) if cols else (512, 320), "bf16", 9)
        want = sp.linear(A, meta, X, act="silu", residual=r, cd_col_major=cols)
        assert torch.equal(sp.linear(A, meta, X, act="silu", residual=r, out=r, cd_col_major=cols), want)


def test_values_that_are_not_finite(sp):
    """NaN and infinities of one token stay with it, and reach the features that keep a weight for them (the product of
    compressed weights multiplies by no others)."""
    W, A, meta, X = layer(sp, 256, 64, 128, "bf16", False, False, 10)
    X[5, 7], X[9, 0] = float("nan"), float("inf")
    y = sp.linear(A, meta, X, cd_col_major=True)
    finite = torch.isfinite(y)
    assert torch.equal(finite[5], W[:, 7] == 0) and torch.equal(finite[9], W[:, 0] == 0)
    assert int((~finite.all(1)).sum()) == 2 and torch.isnan(y[5][W[:, 7] != 0]).all()
    assert torch.equal(torch.isinf(sp.linear(A, meta, X, act="gelu", cd_col_major=True)[9]), W[:, 0] > 0)
    col = torch.ones(64, device="cuda")
    col[3] = float("nan")
    W, A, meta, X = layer(sp, 256, 64, 128, "i8", False, False, 11)
    y = sp.linear(A, meta, X, col_scale=col, cd_col_major=True)
    assert torch.isnan(y[3]).all() and torch.isfinite(y[:3]).all() and torch.isfinite(y[4:]).all()


def test_nothing_to_do(sp):
    _, A, meta, X = layer(sp, 64, 32, 64, "bf16", False, False, 12)
    assert sp.linear(A, meta, X[:0], act="silu", cd_col_major=True).shape == (0, 64)
    W, none = sp.decompress(A, meta), X[:0]
    dX, dW, db = sp.linear_backward(none.new_empty(0, 64), none.new_empty(0, 64), none, W, act="silu", cd_col_major=True)
    assert dX.shape == (0, 64) and dW.shape == W.shape and not dW.any() and db.shape == (64,) and not db.any()


def test_the_first_calls_may_be_captured():
    """A process whose first calls of the operators on rows are made inside a capture (the products load their kernels before: their
    first call outside)."""
    code = (
        "import torch\n"
        "from paper_2104_08378_b200 import binding as sp\n"
        "x = torch.randn(64, 1024, device='cuda').bfloat16(); w = torch.randn(1024, device='cuda').bfloat16()\n"
        "g = torch.cuda.CUDAGraph()\n"
        "with torch.cuda.graph(g):\n"
        "    y, h, s, r = sp.rms_norm(x, w, residual=x, quant='e4m3', with_rstd=True)\n"
        "    a, t = sp.gated_act(x[:, :512], x[:, 512:], quant='i8')\n"
        "    d = sp.rms_norm_backward(x, h, w, r)\n"
        "    e = sp.gated_act_backward(x, x, x)\n"
        "    f = sp.act_backward(x, x, act='gelu')\n"
        "g.replay(); torch.cuda.synchronize()\n"
        "want = sp.rms_norm(x, w, residual=x, quant='e4m3'); assert torch.equal(want[0].view(torch.uint8), y.view(torch.uint8))\n"
        "assert torch.equal(sp.gated_act_backward(x, x, x)[0], e[0]) and torch.equal(sp.rms_norm_backward(x, h, w, r)[1], d[1])\n"
        "assert torch.equal(sp.act_backward(x, x, act='gelu')[1], f[1])\n"
        "print('same')\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and done.stdout.split()[-1:] == ["same"], done


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("act", ACTS)
def test_gradients(sp, t, act):
    for M, N, K, cols, b_rows in ((256, 64, 128, True, False), (320, 208, 144, False, False), (128, 48, 272, True, True), (64, 512, 64, False, True)):
        W, _, meta, X = layer(sp, M, N, K, t, False, b_rows, 13)
        shape = (N, M) if cols else (M, N)
        pre, dy = operand(shape, t, 14), operand(shape, t, 15)
        if t == "f32":                                                      # (there is no mask of the 1:2 pattern)
            with pytest.raises(sp.Sp24Error):
                sp.linear_backward(dy, pre, X, W, act=act, meta=meta, b_row_major=b_rows, cd_col_major=cols)
            meta = None
        dX, dW, db = sp.linear_backward(dy, pre, X, W, act=act, meta=meta, b_row_major=b_rows, cd_col_major=cols)
        slope = act64(pre.double(), act)[1]
        dz = (dy.double() * slope)
        dz = dz if not cols else dz.T                                       # M x N
        x = X.double() if b_rows else X.double().T                          # K x N
        # dz is rounded to the type before the products (TF32 takes 2^-10 of an FP32 value), its slope has 2^-17
        rounding = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -10}[t] + 2.0 ** -17
        dz_bound = (dy.double().abs() if not cols else dy.double().abs().T) * 1.13
        want = W.double().T @ dz
        err = (rounding + (M / 32 + 34) * 2.0 ** -23) * (W.double().abs().T @ dz_bound)
        close(dX, want if b_rows else want.T, t, err if b_rows else err.T)
        want = dz @ x.T * (1 if meta is None else W != 0)
        close(dW, want, t, (rounding + (N / 32 + 34) * 2.0 ** -23) * (dz_bound @ x.T.abs()))
        assert meta is None or not dW[W == 0].any()
        close(db, dz.sum(1), "f32", 2.0 ** -16 * dz_bound.sum(1))


def test_gradients_against_differences(sp):
    """The whole layer, from its formula: inputs, weights and bias moved a little."""
    M, N, K = 32, 16, 32
    W, _, meta, X = layer(sp, M, N, K, "f32", False, False, 16)
    W = W / 4
    b, dy = rand((M,), "f32", 17).double(), rand((N, M), "f32", 18)
    z = X.double() @ W.double().T + b
    dX, dW, db = sp.linear_backward(dy, z.float(), X, W, act="gelu", cd_col_major=True)

    def value(X, W, b):
        return (act64(X @ W.T + b, "gelu")[0] * dy.double()).sum()
    X, W = X.double(), W.double()
    step = 1e-4
    for what, grad, place in ((0, dX, (3, 5)), (0, dX, (15, 31)), (1, dW, tuple((W != 0).nonzero()[7].tolist())), (2, db, (9,))):
        args = [[X, W, b], [X, W, b]]
        for sign, side in ((1, 0), (-1, 1)):
            moved = args[side][what].clone()
            moved[place] += sign * step
            args[side][what] = moved
        slope = float((value(*args[0]) - value(*args[1])) / (2 * step))
        # (TF32 takes 2^-10 of each of up to 32 terms of at most 4 * 4)
        assert abs(slope - float(grad[place])) <= 32 * 16 * 2.0 ** -10 * 0.25, (what, slope, float(grad[place]))


def test_a_feed_forward_layer(sp):
    """norm -> 8-bit product -> gated activation -> 8-bit product with the residual, eager and captured, for int8 and e4m3."""
    rows, K, F = 96, 512, 768
    x, r, w = rand((rows, K), "bf16", 19), rand((rows, K), "bf16", 20), rand((K,), "bf16", 21)
    for quant in ("i8", "e4m3"):
        up, up_vals, up_meta, _ = sp.prune_compress(operand((2 * F, K), quant, 22))
        down, down_vals, down_meta, _ = sp.prune_compress(operand((K, F), quant, 23))
        size = 73.0 if quant == "i8" else 1.0
        up_scale = torch.full((2 * F,), 1 / (size * math.sqrt(K)), device="cuda")
        down_scale = torch.full((K,), 1 / (size * math.sqrt(F)), device="cuda")

        def layer_of(x):
            x8, h, xs, _ = sp.rms_norm(x, w, residual=r, quant=quant)
            gu = sp.linear(up_vals, up_meta, x8, row_scale=up_scale, col_scale=xs, cd="bf16", cd_col_major=True)
            a8, s = sp.gated_act(gu[:, :F], gu[:, F:], quant=quant)
            return sp.linear(down_vals, down_meta, a8, row_scale=down_scale, col_scale=s, residual=h, cd="bf16", cd_col_major=True), h
        y, h = layer_of(x)
        n, _ = rms_norm64(h, w, 1e-6)
        gu = n @ (up.double() * up_scale.double()[:, None]).T
        a = act64(gu[:, :F], "silu")[0] * gu[:, F:]
        want = a @ (down.double() * down_scale.double()[:, None]).T + h.double()
        # Normwise.  Codes are half a step off at most, an rms of 1 / sqrt(12) of a step for int8 (rows whose largest value is about 4 rms: a
        # step of 1/32 rms, 0.9 %) and 2.6 % for e4m3; both factors of a carry the first, a itself another (its largest value is about
        # 12 rms: 2.7 %): at most sqrt(2 * .9^2 + 2.7^2) = 3 % and sqrt(3) * 2.6 = 4.5 % of the product's part, taken twice over.
        part = (want - h.double()).norm()
        assert float((y.double() - want).norm() / part) <= (0.06 if quant == "i8" else 0.09)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            got, _ = layer_of(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, y) and sp.gemm_status() == 0


def test_a_training_step(sp):
    """norm -> linear with GELU and residual, and all its gradients back to the input, against torch's autograd in 64 bits."""
    N, K, M = 64, 256, 256
    x, r, w = rand((N, K), "f16", 24), rand((N, K), "f16", 25), rand((K,), "f16", 26)
    W, vals, meta, _ = sp.prune_compress(rand((M, K), "f16", 27, sigma=1 / 16))
    b, dout = rand((M,), "f32", 28), rand((N, M), "f16", 29)
    y, h, _, rstd = sp.rms_norm(x, w, residual=r, with_rstd=True)
    out, pre = sp.linear(vals, meta, y, bias=b, act="gelu", residual=h, pre=True, cd_col_major=True)
    dy, dW, db = sp.linear_backward(dout, pre, y, W, act="gelu", meta=meta, cd_col_major=True)
    dx, dw = sp.rms_norm_backward(dy, h, w, rstd, dh=dout)
    x64, w64, W64, b64 = (v.double().requires_grad_() for v in (x, w, W, b))
    h64 = x64 + r.double()
    n = h64 / torch.sqrt((h64 * h64).mean(1, keepdim=True) + 1e-6) * w64
    z = n @ W64.T + b64
    ref = z * torch.special.ndtr(z) + h64
    ref.backward(dout.double())
    # Normwise: each of the five values held in FP16 on the way (h, y, pre, dz, dy) is within 2^-11 of itself; a product or a
    # norm passes relative errors of independent elements on without growth, 2^-11 each, slopes with a factor below 2.
    for got, want in ((out, ref), (dx, x64.grad), (dw, w64.grad), (dW, W64.grad * (W64 != 0)), (db, b64.grad)):
        assert float((got.double() - want.detach()).norm() / want.detach().norm()) <= 10 * 2.0 ** -11
