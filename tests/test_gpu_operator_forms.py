"""Forms of the operators around the products that sizes, tiles and strides choose: the activation's gradient in both tiles, every tile shape with the
linear epilogue for dense weights and for tokens in rows of N, gradients whose products take pairs of CTAs, wide norms' gradients with FP32 weights,
offsets past 32 bits, results in place between boundaries, calls at once."""
import threading

import pytest
import torch

from operators_util import act64, close, rand
from test_gpu_linear import check

pytestmark = pytest.mark.gpu
SLOPE = 2.0 ** -17      # of an activation's gradient, as in test_gpu_gated_act.py


@pytest.fixture(scope="module")
def sp():
    from paper_2104_08378_b200 import binding
    return binding


# (64 x 64 tiles, ragged; 128 x 128 where those are 296 or more: 18 x 19 and 32 x 12, ragged too)
@pytest.mark.parametrize("rows,cols", [(64, 64), (72, 136), (200, 264), (1000, 272), (2184, 2312), (4096, 1416)])
@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("act", [None, "gelu", "silu"])
def test_activation_gradient_by_vectors(sp, t, act, rows, cols):
    for pad in (0, 8):
        dy, z = rand((rows, cols), t, 1, pad=pad), rand((rows, cols), t, 2, sigma=2.0, pad=pad)
        want = dy.double() * act64(z.double(), act)[1]
        for tokens_out in (True, False):
            dz, dzt, db = sp.act_backward(dy, z, act=act, cd_col_major=tokens_out)
            close(dz, want, t, SLOPE * dy.double().abs())
            assert torch.equal(dzt, dz.T)
            # (a chain of additions: at most 16 rows of a thread, 16 warps, 64 tiles in eight shares)
            close(db, want.sum(0 if tokens_out else 1), "f32", (SLOPE + 2.0 ** -17) * dy.double().abs().sum(0 if tokens_out else 1))
            alone = sp.act_backward(dy, z, act=act, cd_col_major=tokens_out, transposed=False, bias=False)[0]
            assert torch.equal(alone, dz)


@pytest.mark.parametrize("act", [None, "gelu"])
def test_activation_gradient_of_rows_that_no_vector_divides(sp, act):
    """Without the transpose only the columns have to be whole vectors: the last rows of a tile, in both tiles."""
    for rows, cols in ((131, 200), (2187, 2312)):
        dy, z = rand((rows, cols), "bf16", 3), rand((rows, cols), "bf16", 4)
        out = torch.full((rows + 1, cols), 7.0, dtype=torch.bfloat16, device="cuda")
        dz, none, db = sp.act_backward(dy, z, act=act, transposed=False, out=out[:rows])
        want = dy.double() * act64(z.double(), act)[1]
        close(dz, want, "bf16", SLOPE * dy.double().abs())
        close(db, want.sum(1), "f32", (SLOPE + 2.0 ** -17) * dy.double().abs().sum(1))
        assert none is None and bool((out[rows] == 7).all())


DENSE = ["1x128x1", "2x224x1", "2x224x2", "2x256x1", "2x192x2", "2x240x1", "2x256x2"]
SPARSE_ROWS, DENSE_ROWS = ["1x128x1", "2x224x1", "2x224x2"], ["1x128x1", "2x224x1", "2x224x2", "2x256x1"]


@pytest.mark.parametrize("ab,cd", [("bf16", "bf16"), ("f16", "f32"), ("i8", "bf16"), ("i8", "f32"), ("e4m3", "f16"), ("e5m2", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("dense,b_rows,tile", [(True, False, tile) for tile in DENSE] + [(False, True, tile) for tile in SPARSE_ROWS] +
                         [(True, True, tile) for tile in DENSE_ROWS])
def test_every_tile_of_dense_weights_and_the_other_order(sp, force_tile, ab, cd, dense, b_rows, tile):
    one_byte, tf32 = ab in ("i8", "e4m3", "e5m2"), ab == "f32"
    built = {"2x192x2": not tf32 and ab in ("bf16", "f16", "i8"), "2x240x1": not (one_byte or tf32) and cd == ab, "2x256x2": not tf32,
             "2x256x1": not (tf32 and b_rows)}
    if not built.get(tile, True):
        pytest.skip("not built")
    force_tile(tile)
    for cols in (False, True):
        check(sp, 1120, 704, 512, ab, cd, "silu", 5, dense=dense, b_rows=b_rows, cols=cols)
        check(sp, 1120, 704, 512, ab, cd, "gelu", 6, dense=dense, b_rows=b_rows, cols=cols, residual=False, pre=False)
    check(sp, 544, 480, 288, ab, cd, None, 7, dense=dense, b_rows=b_rows, cols=True, scales=False, pad=16)


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("cols,b_rows", [(True, False), (False, False), (True, True), (False, True)])
def test_gradients_whose_products_take_pairs(sp, t, cols, b_rows):
    M, N, K, act = 2064, 1040, 2096, "gelu" if cols else None
    for m, n, k, rows in ((N, K, M, True), (M, K, N, not b_rows)):
        desc = sp.GemmDesc(sp.DTYPE_CODE[t], sp.DTYPE_CODE[t], m, n, k, k, n if rows else k, n, n, sp.ROW_MAJOR if rows else sp.COL_MAJOR, sp.ROW_MAJOR, sp.ROW_MAJOR, 1)
        assert sp.gemm_plan(desc).startswith("2x")

    def operand(shape, seed):
        x = rand(shape, t, seed)
        return (x.view(torch.int32) & -8192).view(torch.float32) if t == "f32" else x    # TF32: 13 mantissa bits less
    W, X = operand((M, K), 8), operand((K, N) if b_rows else (N, K), 9)
    pre, dy = operand((N, M) if cols else (M, N), 10), operand((N, M) if cols else (M, N), 11)
    dX, dW, db = sp.linear_backward(dy, pre, X, W, act=act, b_row_major=b_rows, cd_col_major=cols)
    assert sp.gemm_status() == 0
    dz, of = dy.double() * act64(pre.double(), act)[1], dy.double().abs() * 1.13
    dz, of = (dz.T, of.T) if cols else (dz, of)                          # M x N
    x = X.double() if b_rows else X.double().T                           # K x N
    # (as in test_gpu_linear.py: dz is rounded to the type, TF32 takes 2^-10 of it; sums of M or N products)
    rounding = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -10}[t] + 2.0 ** -17
    want, err = W.double().T @ dz, (rounding + (M / 32 + 34) * 2.0 ** -23) * (W.double().abs().T @ of)
    close(dX, want if b_rows else want.T, t, err if b_rows else err.T)
    close(dW, dz @ x.T, t, (rounding + (N / 32 + 34) * 2.0 ** -23) * (of @ x.T.abs()))
    close(db, dz.sum(1), "f32", 2.0 ** -16 * of.sum(1))


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("rows,K,pad", [(5, 12296, 0), (300, 14336, 0), (3, 16384, 0), (297, 16384, 8), (151, 14331, 3), (2, 12289, 0), (150, 8200, 0), (160, 9001, 1)])
@pytest.mark.parametrize("w32", [True, False])
def test_gradient_of_wide_norms(sp, t, rows, K, pad, w32):
    h, dy, dh = rand((rows, K), t, 12, pad=pad), rand((rows, K), t, 13, pad=pad), rand((rows, K), t, 15)
    w = rand((K,), "f32" if w32 else t, 14)
    rstd = (1 / torch.sqrt((h.double() ** 2).mean(1) + 1e-5)).float()
    h64, dy64, r = h.double(), dy.double(), rstd.double()[:, None]
    v = dy64 * w.double()
    for residual in (None, dh):
        dx, dw = sp.rms_norm_backward(dy, h, w, rstd, dh=residual)
        add = 0 if residual is None else residual.double()
        terms = (r * v).abs() + r ** 3 * h64.abs() * (v * h64).abs().mean(1, keepdim=True) + (0 if residual is None else add.abs())
        # (as in test_gpu_rms_norm.py: the mean's sum and a few roundings of each term; a column's sum is of at most 300 rows over 148 blocks)
        close(dx, r * v - r ** 3 * h64 * (v * h64).mean(1, keepdim=True) + add, t, 2.0 ** -17 * terms)
        each = dy64 * h64 * r
        close(dw, each.sum(0), "f32", 2.0 ** -17 * each.abs().sum(0))
        for place in ("dy", "h") + (() if residual is None else ("dh",)):
            a = {"dy": dy.clone(), "h": h.clone(), "dh": dh.clone()}
            b = sp.rms_norm_backward(a["dy"], a["h"], w, rstd, dh=None if residual is None else a["dh"], out=a[place])
            assert b[0] is a[place] and torch.equal(b[0], sp.rms_norm_backward(dy, h, w, rstd, dh=residual, out=torch.empty_like(a[place]))[0]) and torch.equal(b[1], dw)


def test_offsets_past_32_bits(sp):
    """Rows of the product's result, of what the activation was applied to and of the residual so far apart that the last lies more than 2^32 elements behind
    the first; rows of the norm's gradient 2^31 + 8 apart."""
    ld = 2 ** 28 + 2 ** 25
    M, N, K = 64, 16, 64
    room = [torch.empty(15 * ld + 64, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    W, X, bias = rand((M, K), "bf16", 16), rand((N, K), "bf16", 17), rand((M,), "f32", 18)
    for cols, m in ((True, 64), (False, 16)):
        _, vals, meta, _ = sp.prune_compress(W[:m])
        shape = (N, m) if cols else (m, N)
        out, pre, res = (v.as_strided(shape, (ld, 1)) for v in room)
        r = rand(shape, "bf16", 19)
        res.copy_(r)
        sp.linear(vals, meta, X, bias=bias[:m], act="silu", residual=res, pre=pre, out=out, cd_col_major=cols)
        want, z = sp.linear(vals, meta, X, bias=bias[:m], act="silu", residual=r, pre=True, cd_col_major=cols)
        assert torch.equal(out, want) and torch.equal(pre, z) and sp.gemm_status() == 0
        sp.linear(vals, meta, X, bias=bias[:m], act="silu", residual=res, out=res, cd_col_major=cols)
        assert torch.equal(res, want)
    del out, pre, res, room
    ld = 2 ** 31 + 8
    dy, h, dh, dx = (torch.empty(ld + 64, dtype=torch.bfloat16, device="cuda").as_strided((2, 64), (ld, 1)) for _ in range(4))
    small = [rand((2, 64), "bf16", 20 + i) for i in range(3)]
    for far, near in zip((dy, h, dh), small):
        far.copy_(near)
    w, rstd = rand((64,), "bf16", 23), torch.tensor([0.75, 1.25], device="cuda")
    got = sp.rms_norm_backward(dy, h, w, rstd, dh=dh, out=dx)
    want = sp.rms_norm_backward(small[0], small[1], w, rstd, dh=small[2])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("rows,K", [(5000, 1001), (5000, 75), (700, 12289), (300, 16391)])
def test_in_place_between_boundaries(sp, rows, K):
    """More rows than there are teams, each of them sharing 16 bytes with the next: in place, the same as apart."""
    x, r, w = rand((rows, K), "bf16", 24), rand((rows, K), "bf16", 25), rand((K,), "bf16", 26)
    y, h, _, rstd = sp.rms_norm(x, w, residual=r, with_rstd=True)
    a, b = x.clone(), r.clone()
    sp.rms_norm(a, w, residual=b, h_out=b, out=a)
    assert torch.equal(a, y) and torch.equal(b, h)
    a = x.clone()
    assert torch.equal(sp.rms_norm(a, w, out=a)[0], sp.rms_norm(x, w)[0])
    dx, dw = sp.rms_norm_backward(y, h, w, rstd, dh=r)
    a = h.clone()
    got = sp.rms_norm_backward(y, a, w, rstd, dh=r, out=a)
    assert torch.equal(a, dx) and torch.equal(got[1], dw)
    for act in ("silu", "gelu"):
        g = sp.gated_act(x, r, act=act)[0]
        for out in (0, 1):
            both = [x.clone(), r.clone()]
            assert torch.equal(sp.gated_act(both[0], both[1], act=act, out=both[out])[0], g)
        dg, du = sp.gated_act_backward(y, x, r, act=act)
        a, b = x.clone(), r.clone()
        sp.gated_act_backward(y, a, b, act=act, dg=b, du=a)
        assert torch.equal(b, dg) and torch.equal(a, du)
        a = y.clone()
        b = x.clone()
        sp.gated_act_backward(a, b, r, act=act, dg=a, du=b)
        assert torch.equal(a, dg) and torch.equal(b, du)


def chain(sp, seed):
    """norm -> linear with GELU -> gated activation to int8 -> gradients, on inputs of the seed."""
    N, K, M = 96, 512, 768
    x, r, w = rand((N, K), "f16", seed), rand((N, K), "f16", seed + 1), rand((K,), "f16", seed + 2)
    W, vals, meta, _ = sp.prune_compress(rand((M, K), "f16", seed + 3, sigma=1 / 16))
    dout, bias = rand((N, M), "f16", seed + 4), rand((M,), "f32", seed + 5)

    def run():
        y, h, _, rstd = sp.rms_norm(x, w, residual=r, with_rstd=True)
        out, pre = sp.linear(vals, meta, y, bias=bias, act="gelu", pre=True, cd_col_major=True)
        codes, scale = sp.gated_act(out[:, :M // 2], out[:, M // 2:], quant="i8")
        dy, dW, db = sp.linear_backward(dout, pre, y, W, act="gelu", meta=meta, cd_col_major=True)
        dx, dw = sp.rms_norm_backward(dy, h, w, rstd, dh=y)
        return y, h, rstd, out, pre, codes, scale, dy, dW, db, dx, dw
    return run


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_calls_at_once(sp):
    """Two threads with a stream each, and two captured graphs replayed at once: what each gives by itself."""
    runs = [chain(sp, 30), chain(sp, 40)]
    want = [[v.clone() for v in run()] for run in runs]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                got = runs[i]()
                torch.cuda.current_stream().synchronize()
                if not same(got, want[i]):
                    wrong.append(i)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
    graphs = []
    for run in runs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = run()
        graphs.append((graph, got, torch.cuda.Stream()))
    for _ in range(5):
        for graph, got, stream in graphs:
            with torch.cuda.stream(stream):
                for v in got:
                    v.zero_()
                graph.replay()
        torch.cuda.synchronize()
        for (_, got, _), expected in zip(graphs, want):
            assert same(got, expected)
    assert sp.gemm_status() == 0
