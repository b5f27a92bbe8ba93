"""The operators around a 2:4-sparse feed-forward layer, as cases that can be timed and compared.

Three operators and their gradients: the root-mean-square norm with the residual's addition, whose result may be the 8-bit
operand of the product that follows (with a scale for each row); the sparse product with scales, bias, activation and
residual in its epilogue; and the gated activation between the two products of a feed-forward layer, again with an 8-bit
result where wanted.  ``run`` computes them in elementary torch operations in 32 bits, or, with ``own``, by the calls of
``paper_2104_08378_b200.binding`` that a user makes.

``listed`` holds the workloads, ``draw`` spreads the same kinds over their whole range, ragged sizes among them.
"""
import math

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "i8": torch.int8, "e4m3": torch.float8_e4m3fn}
BYTES = {"bf16": 2, "f16": 2, "f32": 4, "i8": 1, "e4m3": 1}
LARGEST = {"i8": 127.0, "e4m3": 448.0}
EPS = 1e-5
MOST_VALUES = 8192 * 12288          # of a matrix that the row operators read
MOST_PRODUCT = 16384 * 4096 * 4096  # M * N * K


def listed():
    return [
        # token-by-token decoding of 32 sequences: one norm of a mid-sized model; latency is what counts
        {"name": "norm_decode_bf16", "kind": "norm", "t": "bf16", "rows": 32, "K": 4096, "residual": True, "quant": "", "pad": 0},
        # odd sizes: rows that are no multiple of any vector, in a wider buffer
        {"name": "norm_odd_f16", "kind": "norm", "t": "f16", "rows": 1031, "K": 1531, "residual": True, "quant": "", "pad": 5},
        # prompt processing of the largest layer: residual, norm and the 8-bit operand of the next product in one pass
        {"name": "norm_prefill_e4m3", "kind": "norm", "t": "bf16", "rows": 8192, "K": 12288, "residual": True, "quant": "e4m3", "pad": 0},
        # training: the norm's gradient, with the one that arrives along the residual
        {"name": "norm_backward_bf16", "kind": "norm_backward", "t": "bf16", "rows": 8192, "K": 8192, "residual": True},
        # decoding in the INT8 deployment: weights scaled by row, activations by token
        {"name": "linear_decode_i8", "kind": "linear", "ab": "i8", "cd": "bf16", "M": 4096, "N": 32, "K": 4096, "act": "",
         "bias": True, "residual": True, "tokens_out": True, "pre": False, "b_rows": False},
        # prompt processing, 16 bits: up-projection with bias and GELU
        {"name": "linear_gelu_bf16", "kind": "linear", "ab": "bf16", "cd": "bf16", "M": 16384, "N": 4096, "K": 4096, "act": "gelu",
         "bias": True, "residual": False, "tokens_out": True, "pre": False, "b_rows": False},
        # a ragged product as a training step calls it: what the activation is applied to is kept for the gradient
        {"name": "linear_ragged_f16", "kind": "linear", "ab": "f16", "cd": "f16", "M": 1184, "N": 736, "K": 1008, "act": "silu",
         "bias": True, "residual": True, "tokens_out": False, "pre": True, "b_rows": True},
        # training: all gradients of a linear layer with GELU
        {"name": "linear_backward_bf16", "kind": "linear_backward", "ab": "bf16", "M": 8192, "N": 4096, "K": 2048, "act": "gelu",
         "tokens_out": True},
        # the INT8 feed-forward layer of 512 tokens as a whole: norm, up-projection, gated activation, down-projection
        {"name": "ffn_i8", "kind": "ffn", "t": "bf16", "rows": 512, "K": 4096, "F": 8192, "act": "silu"},
        # decoding: gated activation to the 8-bit operand
        {"name": "gated_decode_e4m3", "kind": "gated", "t": "bf16", "rows": 32, "F": 8192, "act": "silu", "quant": "e4m3"},
        # prompt processing: the same for 8192 tokens
        {"name": "gated_prefill_e4m3", "kind": "gated", "t": "bf16", "rows": 8192, "F": 12288, "act": "silu", "quant": "e4m3"},
        # training: gradients of both factors, ragged
        {"name": "gated_backward_f16", "kind": "gated_backward", "t": "f16", "rows": 4099, "F": 5461, "act": "gelu"},
    ]


def _log(rng, lo, hi, multiple=1):
    """A multiple of `multiple` between lo and hi, even over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi // multiple * multiple, max(multiple, round(v / multiple) * multiple))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_backward", "linear", "linear", "linear_backward", "ffn", "gated", "gated_backward"])
    if kind in ("norm", "norm_backward", "gated", "gated_backward"):
        rows, width = _log(rng, 1, 8192), _log(rng, 64, 12288, rng.choice([1, 8, 64]))
        t = rng.choice(["bf16", "bf16", "f16", "f32"])
        if t == "f32" and rows * width > MOST_VALUES // 4:
            rows = max(1, MOST_VALUES // 4 // width)
        if kind == "norm":
            quant = rng.choice(["", "e4m3"])
            return {"kind": kind, "t": t, "rows": rows, "K": width, "residual": rng.random() < 0.7, "quant": quant,
                    "pad": rng.choice([0, 0, 8, 5])}
        if kind == "norm_backward":
            return {"kind": kind, "t": t, "rows": rows, "K": width, "residual": rng.random() < 0.7}
        act = rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"])
        if kind == "gated":
            return {"kind": kind, "t": t, "rows": rows, "F": width, "act": act, "quant": rng.choice(["", "e4m3"])}
        rows = min(rows, max(1, MOST_VALUES // 2 // width))
        return {"kind": kind, "t": t, "rows": rows, "F": width, "act": act}
    M, K = _log(rng, 128, 16384, 32), _log(rng, 128, 8192, 32)
    if kind == "ffn":
        return {"kind": kind, "t": rng.choice(["bf16", "f16"]), "rows": _log(rng, 32, 1024, 32), "K": _log(rng, 256, 4096, 32),
                "F": _log(rng, 256, 8192, 32), "act": rng.choice(["silu", "gelu"])}
    N = _log(rng, 32, 8192, 32)
    if M * N * K > MOST_PRODUCT // 2:
        N = max(32, MOST_PRODUCT // 2 // (M * K) // 32 * 32)
    act = rng.choice(["", "relu", "gelu", "silu", "gelu_tanh"])
    if kind == "linear_backward":
        N = max(32, N // 2 // 32 * 32)
        return {"kind": kind, "ab": rng.choice(["bf16", "f16"]), "M": M, "N": N, "K": K, "act": act, "tokens_out": rng.random() < 0.7}
    ab = rng.choice(["bf16", "bf16", "f16", "e4m3", "i8"])
    return {"kind": kind, "ab": ab, "cd": ab if BYTES[ab] == 2 else rng.choice(["bf16", "f16"]), "M": M, "N": N, "K": K, "act": act,
            "bias": rng.random() < 0.7, "residual": rng.random() < 0.5, "tokens_out": rng.random() < 0.7, "pre": rng.random() < 0.3,
            "b_rows": rng.random() < 0.15}


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _normal(g, shape, sigma=1.0):
    return torch.randn(shape, generator=g, device="cuda") * sigma


def _activations(g, rows, width, t, pad=0):
    """Rows of activations of type t; with pad, a view of rows that are `pad` longer."""
    full = _normal(g, (rows, width + pad))
    return full.to(DTYPE[t])[:, :width]


def _weights(g, M, K, ab):
    """Weights M x K of which every aligned group of four along K has its two largest magnitudes."""
    w = _normal(g, (M, K), 1.0 / math.sqrt(K))
    if ab == "i8":
        w = (w * (32.0 * math.sqrt(K))).round().clamp_(-127, 127)
    elif ab == "e4m3":
        w = (w * (8.0 * math.sqrt(K))).to(DTYPE[ab]).float()
    else:
        w = w.to(DTYPE[ab]).float()
    groups = w.view(M, K // 4, 4)
    keep = torch.zeros_like(groups).scatter_(2, groups.abs().topk(2, dim=2).indices, 1.0)
    return (groups * keep).view(M, K).to(DTYPE[ab])


def _layer(g, M, K, ab):
    """A layer as a program keeps it: the pruned weights (training keeps them dense, as the plain form reads them) and, for
    the framework's products, their compressed form, laid out once."""
    layer = {"W": _weights(g, M, K, ab)}
    if own:
        from paper_2104_08378_b200 import binding as sp
        layer["vals"], layer["meta"], _ = sp.compress(layer["W"])
    return layer


def _row_scales(g, n, size):
    return (torch.rand(n, generator=g, device="cuda") + 0.5) * size


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case}
    kind = case["kind"]
    if kind in ("norm", "norm_backward"):
        rows, K, t = case["rows"], case["K"], case["t"]
        s["x"] = _activations(g, rows, K, t, case.get("pad", 0))
        s["weight"] = (_normal(g, (K,), 0.1) + 1.0).to(DTYPE[t])
        if kind == "norm":
            s["residual"] = _activations(g, rows, K, t, case["pad"]) if case["residual"] else None
        else:  # what the forward call has left: its input and 1 / rms of each row
            s["rstd"] = (s["x"].float().square().mean(1) + EPS).rsqrt()
            s["dy"] = _activations(g, rows, K, t)
            s["dh"] = _activations(g, rows, K, t) if case["residual"] else None
    elif kind in ("gated", "gated_backward"):
        rows, F, t = case["rows"], case["F"], case["t"]
        s["gu"] = _activations(g, rows, 2 * F, t)  # both halves of an up-projection's result
        if kind == "gated_backward":
            s["dy"] = _activations(g, rows, F, t)
    elif kind == "linear":
        M, N, K, ab = case["M"], case["N"], case["K"], case["ab"]
        s.update(_layer(g, M, K, ab))
        x = _normal(g, (K, N) if case["b_rows"] else (N, K))
        s["X"] = (x * 32).round().clamp_(-127, 127).to(torch.int8) if ab == "i8" else x.to(DTYPE[ab])
        s["bias"] = _normal(g, (M,), 0.5) if case["bias"] else None
        s["residual"] = _activations(g, N if case["tokens_out"] else M, M if case["tokens_out"] else N, case["cd"]) if case["residual"] else None
        if BYTES[ab] == 1:
            s["row_scale"] = _row_scales(g, M, 1.0 / (32 * math.sqrt(K)) if ab == "i8" else 1.0 / (8 * math.sqrt(K)))
            s["col_scale"] = _row_scales(g, N, 1.0 / 32 if ab == "i8" else 1.0)
        else:
            s["row_scale"] = s["col_scale"] = None
    elif kind == "linear_backward":
        M, N, K, ab = case["M"], case["N"], case["K"], case["ab"]
        s["W"] = _weights(g, M, K, ab)
        s["X"] = _activations(g, N, K, ab)
        shape = (N, M) if case["tokens_out"] else (M, N)
        s["pre"] = _activations(g, *shape, ab)
        s["dy"] = _activations(g, *shape, ab)
    else:  # ffn
        rows, K, F, t = case["rows"], case["K"], case["F"], case["t"]
        s["x"], s["residual"] = _activations(g, rows, K, t), _activations(g, rows, K, t)
        s["weight"] = (_normal(g, (K,), 0.1) + 1.0).to(DTYPE[t])
        s["up"], s["down"] = _layer(g, 2 * F, K, "i8"), _layer(g, K, F, "i8")
        s["up_scale"] = _row_scales(g, 2 * F, 1.0 / (32 * math.sqrt(K)))
        s["down_scale"] = _row_scales(g, K, 1.0 / (32 * math.sqrt(F)))
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2104_08378_b200 import binding as sp
    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        y, h, scale, _ = sp.rms_norm(s["x"], s["weight"], eps=EPS, residual=s["residual"], quant=case["quant"] or None)
        return y, h, scale
    if kind == "norm_backward":
        return sp.rms_norm_backward(s["dy"], s["x"], s["weight"], s["rstd"], dh=s["dh"])
    if kind == "linear":
        return sp.linear(s["vals"], s["meta"], s["X"], bias=s["bias"], act=case["act"] or None, residual=s["residual"],
                         row_scale=s["row_scale"], col_scale=s["col_scale"], pre=case["pre"], cd=case["cd"],
                         b_row_major=case["b_rows"], cd_col_major=case["tokens_out"])
    if kind == "linear_backward":
        return sp.linear_backward(s["dy"], s["pre"], s["X"], s["W"], act=case["act"] or None, cd_col_major=case["tokens_out"])
    if kind == "gated":
        F = case["F"]
        return sp.gated_act(s["gu"][:, :F], s["gu"][:, F:], act=case["act"], quant=case["quant"] or None)
    if kind == "gated_backward":
        F = case["F"]
        return sp.gated_act_backward(s["dy"], s["gu"][:, :F], s["gu"][:, F:], act=case["act"])
    F, t = case["F"], case["t"]
    x8, h, x_scale, _ = sp.rms_norm(s["x"], s["weight"], eps=EPS, residual=s["residual"], quant="i8")
    gu = sp.linear(s["up"]["vals"], s["up"]["meta"], x8, row_scale=s["up_scale"], col_scale=x_scale, cd=t, cd_col_major=True)
    a8, a_scale = sp.gated_act(gu[:, :F], gu[:, F:], act=case["act"], quant="i8")
    return sp.linear(s["down"]["vals"], s["down"]["meta"], a8, row_scale=s["down_scale"], col_scale=a_scale, residual=h, cd=t,
                     cd_col_major=True), h


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * math.sqrt(0.5 / math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        p = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + p) + 0.5 * z * (1 - p * p) * c * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _quantised(y, quant):
    """8-bit values of the rows of y and the scale of each."""
    scale = y.abs().amax(1) / LARGEST[quant]
    q = y / torch.where(scale > 0, scale, torch.ones_like(scale))[:, None]
    return (q.round() if quant == "i8" else q).to(DTYPE[quant]), scale


def _norm_plain(x, weight, residual, quant):
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    f = h.float()
    y = f * (f.square().mean(1, keepdim=True) + EPS).rsqrt() * weight.float()
    y, scale = _quantised(y, quant) if quant else (y.to(x.dtype), None)
    return y, (None if residual is None else h), scale


def _linear_plain(W, X, cd, act="", bias=None, residual=None, row_scale=None, col_scale=None, tokens_out=True, b_rows=False):
    z = W.float() @ (X.float() if b_rows else X.float().T)
    if row_scale is not None:
        z = z * row_scale[:, None] * col_scale[None, :]
    if bias is not None:
        z = z + bias[:, None]
    if tokens_out:
        z = z.T
    y = _act(z, act)
    if residual is not None:
        y = y + residual.float()
    return y.to(DTYPE[cd]).contiguous(), z


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        return _norm_plain(s["x"], s["weight"], s["residual"], case["quant"])
    if kind == "norm_backward":
        h, dy, r = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
        dyw = dy * s["weight"].float()
        dx = r * dyw - r * r * r * h * (dyw * h).mean(1, keepdim=True)
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return dx.to(s["x"].dtype), (dy * h * r).sum(0)
    if kind == "linear":
        y, z = _linear_plain(s["W"], s["X"], case["cd"], case["act"], s["bias"], s["residual"], s["row_scale"], s["col_scale"],
                             case["tokens_out"], case["b_rows"])
        return (y, z.to(DTYPE[case["cd"]]).contiguous()) if case["pre"] else y
    if kind == "linear_backward":
        dz = s["dy"].float() * _act_slope(s["pre"].float(), case["act"])
        if not case["tokens_out"]:
            dz = dz.T
        dt = s["W"].dtype
        return (dz @ s["W"].float()).to(dt), (dz.T @ s["X"].float()).to(dt), dz.sum(0)
    if kind == "gated":
        g, u = s["gu"].float().split(case["F"], 1)
        y = _act(g, case["act"]) * u
        return _quantised(y, case["quant"]) if case["quant"] else (y.to(s["gu"].dtype), None)
    if kind == "gated_backward":
        g, u = s["gu"].float().split(case["F"], 1)
        dy, t = s["dy"].float(), s["gu"].dtype
        return (dy * u * _act_slope(g, case["act"])).to(t), (dy * _act(g, case["act"])).to(t)
    x8, h, x_scale = _norm_plain(s["x"], s["weight"], s["residual"], "i8")
    gu, _ = _linear_plain(s["up"]["W"], x8, case["t"], row_scale=s["up_scale"], col_scale=x_scale)
    g, u = gu.float().split(case["F"], 1)
    a8, a_scale = _quantised(_act(g, case["act"]) * u, "i8")
    return _linear_plain(s["down"]["W"], a8, case["t"], residual=h, row_scale=s["down_scale"], col_scale=a_scale)[0], h


# ---- what a pass cannot do without -------------------------------------------------------------------------------------
def _product_bytes(M, K, ab):
    """Compressed weights: half the values and two bits for each."""
    return M * K // 2 * BYTES[ab] + M * K // 8


def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_backward"):
        n, e = case["rows"] * case["K"], BYTES[case["t"]]
        if kind == "norm":
            out = n + 4 * case["rows"] if case["quant"] else n * e
            return {"bytes": n * e * (3 if case["residual"] else 1) + out + case["K"] * e, "flops": 5 * n}
        return {"bytes": n * e * (4 if case["residual"] else 3) + 4 * case["rows"] + case["K"] * (e + 4), "flops": 10 * n}
    if kind in ("gated", "gated_backward"):
        n, e = case["rows"] * case["F"], BYTES[case["t"]]
        if kind == "gated":
            return {"bytes": 2 * n * e + (n + 4 * case["rows"] if case["quant"] else n * e), "flops": 10 * n}
        return {"bytes": 5 * n * e, "flops": 20 * n}
    if kind == "linear":
        M, N, K, e, c = case["M"], case["N"], case["K"], BYTES[case["ab"]], BYTES[case["cd"]]
        outs = 1 + bool(case["residual"]) + bool(case["pre"])
        return {"bytes": _product_bytes(M, K, case["ab"]) + N * K * e + outs * M * N * c + 4 * M * bool(case["bias"]) + (4 * (M + N) if e == 1 else 0),
                "flops": M * N * K}  # half of the weights are zeros
    if kind == "linear_backward":
        M, N, K, e = case["M"], case["N"], case["K"], BYTES[case["ab"]]
        return {"bytes": e * (2 * M * N + 2 * M * K + 2 * N * K) + 4 * M, "flops": 4 * M * N * K}
    rows, K, F, e = case["rows"], case["K"], case["F"], BYTES[case["t"]]
    return {"bytes": _product_bytes(2 * F, K, "i8") + _product_bytes(K, F, "i8") + 4 * rows * K * e + 4 * (2 * F + K) + K * e,
            "flops": 3 * rows * K * F}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------
def _act64(z, act):
    """(act(z), act'(z)) from the functions' definitions: Phi is the normal distribution's."""
    if act == "relu":
        step = torch.heaviside(z, torch.zeros((), dtype=z.dtype, device=z.device))
        return z.clamp(min=0), step
    if act == "silu":
        sig = torch.sigmoid(z)
        return z * sig, sig + z * sig * torch.sigmoid(-z)
    if act == "gelu":
        phi = torch.special.ndtr(z)
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":  # (1 + tanh(v)) / 2 = sigmoid(2 v)
        v2 = math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3)
        sig = torch.sigmoid(v2)
        return z * sig, sig + z * sig * torch.sigmoid(-v2) * math.sqrt(8 / math.pi) * (1 + 0.134145 * z ** 2)
    return z, torch.ones_like(z)


def _scaled64(y, quant):
    scale = torch.linalg.vector_norm(y, ord=math.inf, dim=1) / LARGEST[quant]
    codes = y / scale.clamp(min=1e-300)[:, None]
    return (torch.round(codes) if quant == "i8" else codes), scale


def _norm64(x, weight, residual, quant):
    h = x.double()
    if residual is not None:  # the residual stream is held in the inputs' type: so says the definition
        h = (h + residual.double()).to(x.dtype).double()
    rms = torch.sqrt((h * h).sum(1) / h.shape[1] + EPS)
    y = weight.double()[None, :] * h / rms[:, None]
    y, scale = _scaled64(y, quant) if quant else (y, None)
    return y, (None if residual is None else h), scale


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        return _norm64(s["x"], s["weight"], s["residual"], case["quant"])
    if kind == "norm_backward":
        h, dy, w, r = s["x"].double(), s["dy"].double(), s["weight"].double(), s["rstd"].double()
        n = h * r[:, None]
        v = dy * w
        along = torch.einsum("rk,rk->r", v, n) / h.shape[1]
        dx = (v - n * along[:, None]) * r[:, None]
        return dx if s["dh"] is None else dx + s["dh"].double(), torch.einsum("rk,rk->k", dy, n)
    if kind == "linear":
        x = s["X"].double()
        z = (x.T if case["b_rows"] else x) @ s["W"].double().T  # tokens x features
        if s["row_scale"] is not None:
            z = z * torch.outer(s["col_scale"].double(), s["row_scale"].double())
        if s["bias"] is not None:
            z = z + s["bias"].double()
        if not case["tokens_out"]:
            z = z.T
        y = _act64(z, case["act"])[0]
        if s["residual"] is not None:
            y = y + s["residual"].double()
        return (y, z) if case["pre"] else y
    if kind == "linear_backward":
        dz = s["dy"].double() * _act64(s["pre"].double(), case["act"])[1]
        dz = dz if case["tokens_out"] else dz.T
        return torch.einsum("tm,mk->tk", dz, s["W"].double()), torch.einsum("tm,tk->mk", dz, s["X"].double()), dz.sum(0)
    if kind == "gated":
        F = case["F"]
        y = _act64(s["gu"][:, :F].double(), case["act"])[0] * s["gu"][:, F:].double()
        return _scaled64(y, case["quant"]) if case["quant"] else (y, None)
    if kind == "gated_backward":
        F = case["F"]
        a, slope = _act64(s["gu"][:, :F].double(), case["act"])
        return s["dy"].double() * s["gu"][:, F:].double() * slope, s["dy"].double() * a
    F = case["F"]
    x8, h, x_scale = _norm64(s["x"], s["weight"], s["residual"], "i8")
    gu = (x8 @ s["up"]["W"].double().T) * torch.outer(x_scale, s["up_scale"].double())
    gu = gu.to(s["x"].dtype).double()  # the up-projection's result is held in 16 bits
    a8, a_scale = _scaled64(_act64(gu[:, :F], case["act"])[0] * gu[:, F:], "i8")
    return (a8 @ s["down"]["W"].double().T) * torch.outer(a_scale, s["down_scale"].double()) + h, h
