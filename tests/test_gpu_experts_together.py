"""The experts' operators one after the other, as a layer calls them; captured, on other streams, through either form of the binding, past 32-bit offsets; and a wait that
gives up."""
import pytest
import torch

from experts_util import choice
from operators_util import act64, close, rand

pytestmark = pytest.mark.gpu
E, K, F, T, k = 6, 160, 96, 77, 3


@pytest.fixture(scope="module")
def sp():
    from paper_2104_08378_b200 import binding
    return binding


class Silent:
    """A native part that leaves every call to the Python forms."""
    def __getattr__(self, name):
        return lambda *args: None


@pytest.fixture(params=["native", "python"])
def either(sp, request, monkeypatch):
    if request.param == "python":
        monkeypatch.setattr(sp, "_native", Silent())
    return sp


def pruned(sp, shape, t, seed, sigma):
    W = rand(shape, t, seed, sigma)
    return torch.stack([sp.prune(w) for w in W])


class Layer:
    def __init__(self, sp, t="bf16", align=16):
        self.sp, self.align = sp, align
        self.up, self.down = pruned(sp, (E, 2 * F, K), t, 1, K ** -0.5), pruned(sp, (E, K, F), t, 2, F ** -0.5)
        self.cup, self.cdown = sp.expert_compress(self.up), sp.expert_compress(self.down)
        self.logits, self.x, self.dout = rand((T, E), "f32", 3), rand((T, K), t, 4), rand((T, K), t, 5)
        self.logits[-5:] = float("-inf")   # a padded batch

    def forward(self):
        sp = self.sp
        self.weights, self.experts = sp.route(self.logits, k, score="sigmoid")
        self.order = sp.expert_order(self.experts, E, align=self.align)
        self.xs, _ = sp.expert_gather(self.x, self.order)
        self.gu = sp.expert_linear(*self.cup, self.xs, self.order.offsets)
        self.a, _ = sp.gated_act(self.gu[:, :F], self.gu[:, F:])
        self.y = sp.expert_linear(*self.cdown, self.a, self.order.offsets)
        return sp.expert_combine(self.y, self.order, self.weights, residual=self.x)

    def backward(self):
        sp = self.sp
        dy, dw = sp.expert_combine_backward(self.dout, self.y, self.order, self.weights)
        da, d_down, _ = sp.expert_linear_backward(dy, None, self.a, self.down, self.order.offsets, meta=self.cdown[1], bias=False)
        dgu = torch.zeros_like(self.gu)
        sp.gated_act_backward(da, self.gu[:, :F], self.gu[:, F:], dg=dgu[:, :F], du=dgu[:, F:])
        dxs, d_up, _ = sp.expert_linear_backward(dgu, None, self.xs, self.up, self.order.offsets, meta=self.cup[1], bias=False)
        return sp.expert_combine(dxs, self.order, residual=self.dout), d_up, d_down, sp.route_backward(dw, self.logits, self.experts, score="sigmoid")

    def step(self):
        return (self.forward(),) + self.backward()


def reference(layer):
    """The layer in 64 bits by autograd, with the choice that was made."""
    up, down, logits, x = (v.double().clone().requires_grad_() for v in (layer.up, layer.down, layer.logits, layer.x))
    live = layer.experts >= 0
    at = layer.experts.clamp(min=0).long()
    s = torch.gather(torch.sigmoid(logits), 1, at).masked_fill(~live, 0)
    w = s / s.sum(1, keepdim=True).clamp(min=1e-30)
    out = x.clone()
    for i in range(k):
        gu = torch.einsum("tk,tfk->tf", x, up[at[:, i]])
        a = act64(gu[:, :F], "silu")[0] * gu[:, F:]
        out = out + (w[:, i] * live[:, i])[:, None] * torch.einsum("tf,tkf->tk", a, down[at[:, i]])
    out.backward(layer.dout.double())
    return out.detach(), x.grad, up.grad * (layer.up != 0), down.grad * (layer.down != 0), torch.nan_to_num(logits.grad)


# Every result goes through up to six roundings to bf16 or f16 on its way (rows, gu, a, y, dy, da, dgu, dxs), each half a step of what is rounded: in the norm of a whole
# result that is at most 8 half steps times the factor by which sums of the ways can grow over their result (4 here: sums of k = 3 and the residual's).
@pytest.mark.parametrize("t,half", [("bf16", 2.0 ** -8), ("f16", 2.0 ** -11)])
def test_a_training_step(either, t, half):
    layer = Layer(either, t)
    got = layer.step()
    for name, a, b in zip(("out", "dx", "dup", "ddown", "dlogits"), got, reference(layer)):
        assert torch.isfinite(a).all(), name
        assert float((a.double() - b).norm()) <= 32 * half * float(b.norm()), name
    for dW, W in ((got[2], layer.up), (got[3], layer.down)):
        assert bool((dW[W == 0] == 0).all())
    assert bool((got[4][-5:] == 0).all()) and torch.equal(got[0][-5:], layer.x[-5:]) and torch.equal(got[1][-5:], layer.dout[-5:])


def test_the_order_of_rows_does_not_matter(sp):
    """The same sums with and without room between the experts: a row's products do not depend on where it lies."""
    a, b = Layer(sp, align=1), Layer(sp, align=16)
    assert torch.equal(a.forward(), b.forward())


def test_both_forms_of_the_binding_agree(sp, monkeypatch):
    native = [v.clone() for v in Layer(sp).step()]
    i8 = (rand((4, 64, 128), "f32", 9) * 40).clamp(-127, 127).to(torch.int8)
    vals, meta = sp.expert_compress(i8)
    X, off, rs, cs = (rand((50, 128), "f32", 10) * 40).clamp(-127, 127).to(torch.int8), torch.tensor([0, 3, 3, 40, 50], dtype=torch.int32, device="cuda"), rand(
        (4, 64), "f32", 11), rand((50,), "f32", 12)
    x = rand((30, 200), "f16", 13)

    def calls():
        order = sp.expert_order(choice(30, 9, 4, 1, 0.2), 9, align=16)
        return [*sp.expert_linear(vals, meta, X, off, row_scale=rs, col_scale=cs, act="gelu", pre=True, bias=rs, residual=torch.ones((50, 64), dtype=torch.float16, device="cuda"), cd="f16"),
                *sp.expert_gather(x, order, scale=x[:, 0].float().contiguous()), *order, *sp.route(x, 4, groups=5, top_groups=2, group_score="top2", bias=x[0].float()),
                *sp.expert_linear_backward(rand((48, 32), "f16", 1), rand((48, 32), "f16", 2), rand((48, 64), "f16", 3), rand((2, 32, 64), "f16", 4),
                                           torch.tensor([0, 16, 48], dtype=torch.int32, device="cuda"), act="silu")]
    native += [v.clone() for v in calls()]
    monkeypatch.setattr(sp, "_native", Silent())
    python = list(Layer(sp).step()) + calls()
    for i, (a, b) in enumerate(zip(native, python)):
        assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a, b), i


def test_given_results_are_returned(either):
    sp = either
    order = sp.expert_order(choice(5, 4, 2, 1), 4)
    x, y, out = rand((5, 64), "bf16", 1), rand((10, 64), "bf16", 2), torch.empty((10, 64), dtype=torch.bfloat16, device="cuda")
    assert sp.expert_gather(x, order, out=out)[0] is out
    w = rand((5, 2), "f32", 3)
    assert sp.expert_combine_backward(x, y, order, w, out=out)[0] is out
    sums = torch.empty_like(x)
    assert sp.expert_combine(y, order, w, out=sums) is sums


def refused(sp, status, fn, *args, **kwargs):
    with pytest.raises(sp.Sp24Error) as e:
        fn(*args, **kwargs)
    assert e.value.status == status, (fn, e.value)


def test_refusals(either):
    sp = either
    x, l = rand((5, 64), "bf16", 1), rand((5, 16), "f32", 2)
    w, e = sp.route(l, 3)
    order = sp.expert_order(e, 16)
    y = rand((15, 64), "bf16", 3)
    refused(sp, 3, sp.route, l, 17)
    refused(sp, 3, sp.route, l, 0)
    refused(sp, 3, sp.route, l, 3, groups=5)
    refused(sp, 3, sp.route, l, 5, groups=4, top_groups=1)
    refused(sp, 3, sp.route, l, 3, bias=l[0, :8])
    refused(sp, 2, sp.route, l, 3, bias=l[0].half())
    refused(sp, 6, sp.route, l, 3, score="tanh")
    refused(sp, 6, sp.route, l, 3, group_score="mean")
    refused(sp, 6, sp.route, l, 3, bias=l[0].cpu())
    refused(sp, 4, sp.route, l.T, 3)
    refused(sp, 3, sp.route_backward, w, l[:4], e)
    refused(sp, 2, sp.route_backward, w.half(), l, e)
    refused(sp, 2, sp.route_backward, w, l, e.long())
    refused(sp, 2, sp.expert_order, e.long(), 16)
    refused(sp, 4, sp.expert_order, e.T, 16)
    refused(sp, 3, sp.expert_order, e, 0)
    refused(sp, 3, sp.expert_order, e, 16, align=0)
    refused(sp, 3, sp.expert_gather, x[:4], order)
    refused(sp, 3, sp.expert_gather, x, order, scale=w[:, 0].contiguous()[:4])
    refused(sp, 4, sp.expert_gather, rand((64, 5), "bf16", 1).T, order)
    refused(sp, 3, sp.expert_combine, y[:14], order, w)
    refused(sp, 3, sp.expert_combine, y, order, w[:4])
    refused(sp, 2, sp.expert_combine, y, order, w, residual=x.half())
    refused(sp, 6, sp.expert_combine, y, order._replace(position=order.position.cpu()), w)
    refused(sp, 3, sp.expert_combine_backward, x, y[:14], order, w)
    refused(sp, 2, sp.expert_combine_backward, x, y.half(), order, w)
    W = pruned(sp, (2, 32, 64), "bf16", 4, 1.0)
    vals, meta = sp.expert_compress(W)
    off = torch.tensor([0, 8, 15], dtype=torch.int32, device="cuda")
    refused(sp, 3, sp.expert_linear, vals, meta, y[:, :32].contiguous(), off)
    refused(sp, 3, sp.expert_linear, vals, meta, y, off[:2])
    refused(sp, 2, sp.expert_linear, vals, meta, y, off.long())
    refused(sp, 3, sp.expert_linear, vals, meta[:1], y, off)
    refused(sp, 1, sp.expert_linear, vals, None, y, off)
    refused(sp, 4, sp.expert_linear, vals.transpose(0, 1).contiguous().transpose(0, 1), meta, y, off)
    refused(sp, 2, sp.expert_linear, vals, meta, y.half(), off)
    refused(sp, 2, sp.expert_linear, vals, meta, y, off, cd="f16")
    refused(sp, 3, sp.expert_linear, vals, meta, y, off, bias=torch.zeros(32, device="cuda"))
    refused(sp, 6, sp.expert_linear, vals, meta, y, off, col_scale=torch.zeros(15, device="cuda"))
    refused(sp, 6, sp.expert_linear, vals, meta, y, off, act="swish")
    refused(sp, 3, sp.expert_linear, vals, meta, y, off, residual=y)
    refused(sp, 3, sp.expert_linear_backward, y, None, y, W, off)
    refused(sp, 1, sp.expert_linear_backward, y[:, :32].contiguous(), None, y, W, off, act="gelu")
    refused(sp, 3, sp.expert_linear_backward, y[:, :32].contiguous(), None, y, W, off, meta=meta[:1])
    refused(sp, 2, sp.expert_linear_backward, y[:, :32].float(), None, y.float(), W.float(), off)


def test_weights_with_longer_rows(either):
    """Leading dimensions of the stacks that are longer than their rows."""
    sp = either
    W = pruned(sp, (3, 48, 64), "f16", 1, 1.0)
    vals, meta = sp.expert_compress(W)
    room, wide = torch.zeros((3, 48, 48), dtype=torch.float16, device="cuda"), torch.zeros((3, 48, 80), dtype=torch.float16, device="cuda")
    room[:, :, :32], wide[:, :, :64] = vals, W
    X, off = rand((32, 64), "f16", 2), torch.tensor([0, 16, 16, 32], dtype=torch.int32, device="cuda")
    assert torch.equal(sp.expert_linear(room[:, :, :32], meta, X, off), sp.expert_linear(vals, meta, X, off))
    assert torch.equal(sp.expert_linear(wide[:, :, :64], None, X, off, a_is_dense=True), sp.expert_linear(W, None, X, off, a_is_dense=True))
    dy = rand((32, 48), "f16", 3)
    for a, b in zip(sp.expert_linear_backward(dy, None, X, wide[:, :, :64], off), sp.expert_linear_backward(dy, None, X, W, off)):
        assert torch.equal(a, b)
    for a, b in zip(sp.expert_compress(wide[:, :, :64]), (vals, meta)):
        assert torch.equal(a, b)


def test_captured_and_replayed(sp):
    """Forward and backward in a graph, replayed over new logits and rows, beside another graph of the same calls and eager ones on another stream."""
    layer, other = Layer(sp), Layer(sp)
    layer.step()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graphs = []
    with torch.cuda.stream(stream):
        for one in (layer, other):
            one.step()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                results = one.step()
            graphs.append((graph, results))
    for seed in (21, 22):
        for one in (layer, other):
            one.logits[:-5] = rand((T - 5, E), "f32", seed)
            one.x.copy_(rand((T, K), "bf16", seed + 5))
        torch.cuda.synchronize()
        for graph, _ in graphs:
            graph.replay()
        eager = Layer(sp)
        eager.logits, eager.x = layer.logits, layer.x
        want = eager.step()
        torch.cuda.synchronize()
        for _, results in graphs:
            for a, b in zip(results, want):
                assert torch.equal(a, b)


def test_two_streams_at_once(sp):
    layers = [Layer(sp), Layer(sp)]
    layers[1].x.mul_(2.0)
    want = [[v.clone() for v in layer.step()] for layer in layers]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for layer, stream in zip(layers, streams):
            with torch.cuda.stream(stream):
                got.append(layer.step())
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(u, v) for u, v in zip(a, b))


@pytest.mark.parametrize("tile", ["1x128x1", "2x128x1"])
def test_no_expert_has_rows(sp, force_tile, tile):
    """Offsets that name none of the rows there are: nothing is written but the weights' gradients, which are zeros."""
    W = pruned(sp, (4, 256, 256), "bf16", 1, 1.0)
    vals, meta = sp.expert_compress(W)
    X, off = rand((900, 256), "bf16", 2), torch.zeros(5, dtype=torch.int32, device="cuda")
    out = torch.full((900, 256), 7.0, dtype=torch.bfloat16, device="cuda")
    force_tile(tile)
    sp.expert_linear(vals, meta, X, off, out=out)
    assert bool((out == 7).all())
    _, dW, db = sp.expert_linear_backward(X, None, X, W, off)
    assert bool((dW == 0).all()) and bool((db == 0).all()) and sp.gemm_status() == 0


@pytest.mark.parametrize("tile", ["1x64x1", "2x224x1"])
def test_an_expired_wait_is_reported(sp, force_tile, tile):
    """A k-block that never comes: the kernel returns within the limit, and the record says so."""
    W = pruned(sp, (2, 256, 1024), "bf16", 1, 1.0)
    vals, meta = sp.expert_compress(W)
    X, off = rand((600, 1024), "bf16", 2), torch.tensor([0, 300, 600], dtype=torch.int32, device="cuda")
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    force_tile(tile)
    want = sp.expert_linear(vals, meta, X, off, ws=ws)
    sp.set_fault_hooks(1000000, True)
    try:
        sp.expert_linear(vals, meta, X, off, ws=ws)
        assert sp.gemm_status(ws) == 9
    finally:
        sp.set_fault_hooks(0, False)
    assert torch.equal(sp.expert_linear(vals, meta, X, off, ws=ws), want) and sp.gemm_status(ws) == 0


def test_offsets_past_32_bits(sp):
    """Rows whose elements and bytes lie behind 2^31 and 2^32."""
    T_, K_, k_ = 36000, 8192, 8
    experts = torch.arange(k_, dtype=torch.int32, device="cuda").expand(T_, k_).contiguous()
    order = sp.expert_order(experts, k_)
    x = rand((T_, K_), "f32", 1).to(torch.bfloat16)
    rows, _ = sp.expert_gather(x, order)
    assert rows.numel() > 2 ** 31
    for r in (0, T_ - 1, T_, 8 * T_ - 3, 8 * T_ - 1):
        assert torch.equal(rows[r], x[r % T_])
    w = torch.full((T_, k_), 0.25, device="cuda")
    total = sp.expert_combine(rows, order, w)
    assert torch.equal(total, 2 * x)
    _, dw = sp.expert_combine_backward(x, rows, order, w, out=rows)
    assert torch.equal(rows[8 * T_ - 1], (0.25 * x[T_ - 1].float()).to(torch.bfloat16))
    norm = (x[-1].double() ** 2).sum()
    assert abs(float(dw[T_ - 1, 7].double() - norm)) <= 2.0 ** -16 * float(norm)
    del rows, total, dw
    W = pruned(sp, (k_, 8192, 64), "bf16", 2, 0.1)
    vals, meta = sp.expert_compress(W)
    X = rand((8 * T_, 64), "bf16", 3)
    D = sp.expert_linear(vals, meta, X, order.offsets)
    assert D.numel() > 2 ** 31 and sp.gemm_status() == 0
    for r in (5, 3 * T_ + 1, 8 * T_ - 1):
        z = W[r // T_].double() @ X[r].double()
        close(D[r], z, "bf16", 40 * 2.0 ** -23 * (W[r // T_].double().abs() @ X[r].double().abs()))


