"""The root-mean-square norm and its gradient against plain implementations in 64 bits: types, sizes, strides and alignments,
the residual, 8-bit results, rows that are zero or not finite, refusals, captured calls."""
import pytest
import torch

from operators_util import DTYPE, check_codes, close, rand, rms_norm64

pytestmark = pytest.mark.gpu
EPS = 1e-5
# FP32 arithmetic of n: the sum of squares and its tree (a term passes at most 64 additions at these lengths: 32 in a thread's
# chain, 10 in the tree, the rest slack), rsqrtf (2^-22), three products: below 2^-17 of the value, taken for each element.
ARITHMETIC = 2.0 ** -17


@pytest.fixture(scope="module")
def sp():
    from paper_2104_08378_b200 import binding
    return binding


SHAPES = [(1, 1), (1, 7), (3, 8), (5, 32), (2, 33), (7, 255), (33, 256), (9, 1000), (4, 1024), (6, 1531), (3, 4096), (2, 8200), (5, 12288),
          (2, 16391), (1, 32768), (1, 32776), (1, 70001)]


@pytest.mark.parametrize("t", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,K", SHAPES)
def test_norm(sp, t, rows, K):
    for pad, residual, w32, offset in ((0, True, False, 0), (8, False, True, 0), (5, True, True, 1), (3, False, False, 1)):
        x = rand((rows, K + offset), t, 1, pad=pad)[:, offset:]
        r = rand((rows, K), t, 2, pad=pad) if residual else None
        w = rand((K,), "f32" if w32 else t, 3)
        y, h, scale, rstd = sp.rms_norm(x, w, eps=EPS, residual=r, with_rstd=True)
        ref = x if r is None else (x.double() + r.double()).to(DTYPE[t])
        assert scale is None and (h is None if r is None else torch.equal(h, ref))
        n, rstd64 = rms_norm64(ref, w, EPS)
        close(y, n, t, ARITHMETIC * n.abs())
        close(rstd, rstd64, "f32", ARITHMETIC * rstd64)
        n, _ = rms_norm64(ref, None, EPS)
        close(sp.rms_norm(x, eps=EPS, residual=r)[0], n, t, ARITHMETIC * n.abs())


@pytest.mark.parametrize("t", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("quant", ["i8", "e4m3", "e5m2"])
@pytest.mark.parametrize("rows,K", [(1, 1), (3, 17), (65, 128), (7, 1531), (4, 4096), (3, 12288), (2, 33000)])
def test_eight_bit_results(sp, t, quant, rows, K):
    for residual, pad in ((True, 0), (False, 3)):
        x, w = rand((rows, K), t, 4, pad=pad), rand((K,), t, 5)
        r = rand((rows, K), t, 6) if residual else None
        x[rows // 2] = 0
        if r is not None:
            r[rows // 2] = 0
        y, h, scale, rstd = sp.rms_norm(x, w, eps=EPS, residual=r, quant=quant)
        assert y.dtype == DTYPE[quant] and rstd is None
        n, _ = rms_norm64(x if h is None else h, w, EPS)
        check_codes(y, scale, n, quant, ARITHMETIC)
        assert float(scale[rows // 2]) == 0 and not y[rows // 2].double().any()


@pytest.mark.parametrize("quant", [None, "i8", "e4m3", "e5m2"])
def test_rows_that_are_not_finite_leave_the_others_alone(sp, quant):
    x, w = rand((6, 520), "bf16", 7), rand((520,), "bf16", 8)
    clean = sp.rms_norm(x, w, eps=EPS, quant=quant)
    x[1, 17], x[3, 500], x[4, 0] = float("nan"), float("inf"), float("-inf")
    y, _, scale, _ = sp.rms_norm(x, w, eps=EPS, quant=quant)
    for row in (0, 2, 5):
        assert torch.equal(y[row].view(torch.uint8), clean[0][row].view(torch.uint8))
        assert quant is None or torch.equal(scale[row], clean[2][row])
    if quant is None:
        assert torch.isnan(y[1]).all() and torch.isnan(y[3, 500]) and torch.isnan(y[4, 0])
        assert not y[3].double().nan_to_num().any()
    else:
        assert torch.isnan(scale[[1, 3, 4]]).all()
        codes = y[[1, 3, 4]].float()
        assert not codes.any() if quant == "i8" else torch.isnan(codes).all()


def test_in_place_and_into_given_tensors(sp):
    x, r, w = rand((9, 1000), "bf16", 9), rand((9, 1000), "bf16", 10), rand((1000,), "bf16", 11)
    y, h, _, _ = sp.rms_norm(x, w, residual=r)
    for first in (True, False):                      # h in place of x or of the residual, y in place of the other
        a, b = x.clone(), r.clone()
        y2, h2, _, _ = sp.rms_norm(a, w, residual=b, h_out=a if first else b, out=b if first else a)
        assert torch.equal(y2, y) and torch.equal(h2, h) and (h2 is a) == first
    a = x.clone()
    assert torch.equal(sp.rms_norm(a, w, out=a)[0], sp.rms_norm(x, w)[0])
    wide = torch.full((9, 1100), 7.0, dtype=torch.bfloat16, device="cuda")
    sp.rms_norm(x, w, residual=r, out=wide[:, 50:1050])
    assert torch.equal(wide[:, 50:1050], y) and bool((wide[:, :50] == 7).all()) and bool((wide[:, 1050:] == 7).all())


@pytest.mark.parametrize("t", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,K", SHAPES + [(1300, 64), (700, 1531), (601, 5000)])
def test_gradient(sp, t, rows, K):
    for residual, w32, pad in ((True, False, 0), (False, True, 3)):
        h, dy = rand((rows, K), t, 12, pad=pad), rand((rows, K), t, 13)
        w, dh = rand((K,), "f32" if w32 else t, 14), rand((rows, K), t, 15, pad=pad) if residual else None
        rstd = (1 / torch.sqrt((h.double() ** 2).mean(1) + EPS)).float()
        dx, dw = sp.rms_norm_backward(dy, h, w, rstd, dh=dh)
        h64, dy64, r = h.double(), dy.double(), rstd.double()[:, None]
        v = dy64 * w.double()
        along = (v * h64).mean(1, keepdim=True)
        want = r * v - r ** 3 * h64 * along + (0 if dh is None else dh.double())
        # FP32: the mean's sum is off by 2^-17 of the sum of magnitudes, the rest by a few roundings of each term
        terms = (r * v).abs() + r ** 3 * h64.abs() * (v * h64).abs().mean(1, keepdim=True) + (0 if dh is None else dh.double().abs())
        close(dx, want, t, 2.0 ** -17 * terms)
        each = dy64 * h64 * r
        # ... and a column's sum passes at most rows additions, pairs of 2^-24, of which 2^-17 covers 128 in a chain
        close(dw, each.sum(0), "f32", 2.0 ** -17 * each.abs().sum(0))
        again = sp.rms_norm_backward(dy, h, w, rstd, dh=dh)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
        assert sp.rms_norm_backward(dy, h, None, rstd, dh=dh)[1] is None
        a = dy.clone()
        assert torch.equal(sp.rms_norm_backward(a, h, w, rstd, dh=dh, out=a)[0], dx)


def test_gradient_against_differences(sp):
    x, r, w = rand((3, 96), "f32", 16).double(), rand((3, 96), "f32", 17).double(), rand((96,), "f32", 18).double()
    dy, dh = rand((3, 96), "f32", 19), rand((3, 96), "f32", 20)

    def value(x, w):                                       # what the gradients are of, from the formula
        n, _ = rms_norm64(x + r, w, EPS)
        return (n * dy.double()).sum() + ((x + r) * dh.double()).sum()
    _, h, _, rstd = sp.rms_norm(x.float(), w.float(), eps=EPS, residual=r.float(), with_rstd=True)
    dx, dw = sp.rms_norm_backward(dy, h, w.float(), rstd, dh=dh)
    for k in (0, 41, 95):
        step = torch.zeros_like(x)
        step[1, k] = 1e-4
        assert abs(float((value(x + step, w) - value(x - step, w)) / 2e-4 - dx[1, k])) < 2e-5   # step^2 and FP32's roundings of values up to 10
        step = torch.zeros_like(w)
        step[k] = 1e-4
        assert abs(float((value(x, w + step) - value(x, w - step)) / 2e-4 - dw[k])) < 2e-5


def test_no_rows(sp):
    x, w = rand((0, 64), "bf16", 1), rand((64,), "bf16", 2)
    y, h, scale, _ = sp.rms_norm(x, w, residual=x, quant="i8")
    assert y.shape == h.shape == (0, 64) and scale.shape == (0,)
    dx, dw = sp.rms_norm_backward(x, x, w, torch.empty(0, device="cuda"))
    assert dx.shape == (0, 64) and not dw.any()


def test_captured_and_on_another_stream(sp):
    x, r, w = rand((40, 1040), "f16", 21), rand((40, 1040), "f16", 22), rand((1040,), "f16", 23)
    dy = rand((40, 1040), "f16", 24)
    side = torch.cuda.Stream()

    def step():
        y, h, scale, rstd = sp.rms_norm(x, w, residual=r, quant="e4m3", with_rstd=True)
        return (y, h, scale) + sp.rms_norm_backward(dy, h, w, rstd, dh=x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        want = [v.clone() for v in step()]
    side.synchronize()
    graphs = []
    for _ in range(2):                                      # two graphs: each has its own workspace
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step()
        graphs.append((graph, got))
    for graph, got in graphs:
        graph.replay()
    torch.cuda.synchronize()
    for _, got in graphs:
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))
    x.copy_(rand((40, 1040), "f16", 25))
    want = [v.clone() for v in step()]
    graphs[0][0].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(graphs[0][1], want))


def test_offsets_past_32_bits(sp):
    """The last row of a view whose rows lie 2^31 + 8 elements apart."""
    ld = 2 ** 31 + 8
    flat = torch.empty(ld + 64, dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((2, 64), (ld, 1))
    x.copy_(rand((2, 64), "bf16", 26))
    w = rand((64,), "bf16", 27)
    n, _ = rms_norm64(x, w, 1e-6)
    close(sp.rms_norm(x, w)[0], n, "bf16", ARITHMETIC * n.abs())


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("K", [8, 64, 128, 264, 512, 1024, 1096, 4096, 8192, 12288, 16384, 20000])
def test_a_row_does_not_depend_on_the_others(sp, t, K):
    """The same bits for a row by itself, among a few and among many (other numbers of teams, vectors to a thread and blocks)."""
    x, r, w = rand((1200, K), t, 28), rand((1200, K), t, 29), rand((K,), t, 30)
    y, _, _, rstd = sp.rms_norm(x, w, residual=r, with_rstd=True)
    q, _, scale, _ = sp.rms_norm(x, w, quant="i8")
    dx, _ = sp.rms_norm_backward(r, x, w, rstd, dh=y)
    for rows in (slice(0, 1), slice(7, 8), slice(100, 260), slice(600, 1199)):
        a = sp.rms_norm(x[rows], w, residual=r[rows], with_rstd=True)
        b = sp.rms_norm(x[rows], w, quant="i8")
        assert torch.equal(a[0], y[rows]) and torch.equal(a[3], rstd[rows]) and torch.equal(b[0], q[rows]) and torch.equal(b[2], scale[rows])
        assert torch.equal(sp.rms_norm_backward(r[rows], x[rows], w, rstd[rows], dh=y[rows])[0], dx[rows])


@pytest.mark.parametrize("t", ["f16", "bf16"])
def test_small_and_large_values(sp, t):
    """The sum with the residual is rounded once, subnormal values and overflows to infinity included; norms of rows of subnormals, and of rows whose
    squares leave FP32."""
    x, r = rand((4, 264), t, 31), rand((4, 264), t, 32)
    tiny = 2.0 ** -20 if t == "f16" else 2.0 ** -130
    x[0], r[0] = x[0] * tiny, r[0] * tiny
    x[1, :8], r[1, :8] = (60000.0, 60000.0) if t == "f16" else (3e38, 3e38)
    y, h, _, rstd = sp.rms_norm(x, residual=r, eps=0.0 if t == "f16" else 1e-30, with_rstd=True)
    assert torch.equal(h, (x.double() + r.double()).to(DTYPE[t])) and torch.isinf(h[1, :8]).all()
    n, _ = rms_norm64(h[[0, 2, 3]], None, 0.0 if t == "f16" else 1e-30)
    close(y[[0, 2, 3]], n, t, ARITHMETIC * n.abs() + (0 if t == "f16" else 1e-20))
    if t == "bf16":
        big = torch.full((1, 264), 1e30, dtype=torch.bfloat16, device="cuda")
        y, _, scale, _ = sp.rms_norm(big, quant="i8")
        assert float(scale) == 0 and not sp.rms_norm(big)[0].any()
