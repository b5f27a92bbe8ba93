"""A feed-forward layer of 2:4-sparse experts, as cases that can be timed and compared.

The operators: the routing of tokens to experts (scores by softmax or sigmoid, a bias for balance, groups, the k best,
renormalised weights) with its gradient, and the order of the rows by experts that it leads to; the gathering of the tokens'
rows in that order and the weighted sum back, with their gradients; and the product of every expert's rows with its own
weights, with scales for each channel and each row, bias, activation and residual, and its gradients.  ``run`` computes them
in elementary torch operations in 32 bits (64 where the choice of an expert hangs on it), or, with ``own``, by the calls of
``paper_2104_08378_b200.binding`` that a user makes.

``listed`` holds the workloads, ``draw`` spreads the same kinds over their whole range, ragged sizes among them.
"""
import math
import random

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "i8": torch.int8, "e4m3": torch.float8_e4m3fn}
BYTES = {"bf16": 2, "f16": 2, "f32": 4, "i8": 1, "e4m3": 1}
EPS = 1e-5
MOST_VALUES = 8192 * 8 * 4096           # of a matrix of rows in the experts' order
MOST_PRODUCT = 16384 * 8192 * 4096      # rows * M * K
MOST_WEIGHTS = 16 * 8192 * 4096         # of all experts


def listed():
    return [
        # token-by-token decoding of 32 sequences: the routing of one layer and the order of its rows; latency is what counts
        {"name": "route_decode_bf16", "kind": "route", "t": "bf16", "T": 32, "E": 64, "k": 8, "score": "softmax", "bias": False, "groups": 1,
         "top_groups": 1, "group_score": "max", "renorm": True, "scale": 1.0, "masked": False, "align": 1},
        # prompt processing with many experts in groups, balanced by a bias
        {"name": "route_prefill_f32", "kind": "route", "t": "f32", "T": 16384, "E": 256, "k": 8, "score": "sigmoid", "bias": True, "groups": 8,
         "top_groups": 4, "group_score": "top2", "renorm": True, "scale": 2.5, "masked": False, "align": 1},
        # training: the router's gradient, where the softmax over all experts is kept as it is
        {"name": "route_backward_bf16", "kind": "route_backward", "t": "bf16", "T": 16384, "E": 128, "k": 4, "score": "softmax", "renorm": False,
         "scale": 1.0, "masked": False},
        # prompt processing: 8-bit rows and their scales in the experts' order, each token to eight experts
        {"name": "gather_prefill_e4m3", "kind": "gather", "t": "e4m3", "T": 8192, "K": 4096, "E": 64, "k": 8, "align": 1, "dropped": False},
        # odd sizes: rows that are no multiple of any vector, some tokens of a padded batch without experts
        {"name": "combine_odd_f16", "kind": "combine", "t": "f16", "T": 1031, "K": 1531, "E": 9, "k": 3, "align": 1, "dropped": True,
         "weights": True, "residual": True},
        # training: gradients of the weighted sum
        {"name": "combine_backward_bf16", "kind": "combine_backward", "t": "bf16", "T": 8192, "K": 4096, "E": 64, "k": 4, "align": 16,
         "dropped": False},
        # decoding in the INT8 deployment: 64 rows over 32 experts, weights scaled by channel, rows by token
        {"name": "linear_decode_i8", "kind": "linear", "ab": "i8", "cd": "bf16", "E": 32, "M": 4096, "K": 4096, "rows": 64, "skew": 1.0, "act": "",
         "bias": False, "residual": False, "pre": False, "dense": False},
        # prompt processing, 16 bits: up-projection with bias and GELU
        {"name": "linear_prefill_bf16", "kind": "linear", "ab": "bf16", "cd": "bf16", "E": 16, "M": 8192, "K": 4096, "rows": 16384, "skew": 0.3,
         "act": "gelu", "bias": True, "residual": False, "pre": False, "dense": False},
        # ragged, as a training step calls it: what the activation is applied to is kept for the gradient
        {"name": "linear_ragged_f16", "kind": "linear", "ab": "f16", "cd": "f16", "E": 9, "M": 1184, "K": 1008, "rows": 2311, "skew": 1.0,
         "act": "silu", "bias": True, "residual": True, "pre": True, "dense": False},
        # training: all gradients of the experts' up-projection
        {"name": "linear_backward_bf16", "kind": "linear_backward", "ab": "bf16", "E": 8, "M": 4096, "K": 2048, "rows": 8192, "skew": 0.3,
         "act": "gelu"},
        # the INT8 layer of 32 decoded tokens as a whole: norm, routing, gathering, two products with a gated activation between, sum
        {"name": "layer_decode_i8", "kind": "layer", "t": "bf16", "quant": True, "T": 32, "K": 2048, "F": 1408, "E": 32, "k": 4, "act": "silu"},
        # a training step of such a layer in 16 bits, forward and backward
        {"name": "layer_train_bf16", "kind": "layer_train", "t": "bf16", "T": 2048, "K": 2048, "F": 1408, "E": 8, "k": 2, "act": "silu"},
    ]


def _log(rng, lo, hi, multiple=1):
    """A multiple of `multiple` between lo and hi, even over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi // multiple * multiple, max(multiple, round(v / multiple) * multiple))


def draw(rng):
    kind = rng.choice(["route", "route", "route_backward", "gather", "combine", "combine_backward", "linear", "linear", "linear", "linear_backward",
                       "layer", "layer_train"])
    if kind in ("route", "route_backward"):
        groups = rng.choice([1, 1, 2, 4, 8]) if kind == "route" else 1
        E = _log(rng, 8, 256, groups)
        E = max(E, 2 * groups)
        top_groups = rng.randint(1, groups)
        k = rng.randint(1, min(8, top_groups * (E // groups)))
        case = {"kind": kind, "t": rng.choice(["bf16", "f16", "f32"]), "T": _log(rng, 1, 16384), "E": E, "k": k,
                "score": rng.choice(["softmax", "sigmoid"]), "renorm": rng.random() < 0.6, "scale": rng.choice([1.0, 2.5]),
                "masked": rng.random() < 0.3}
        if kind == "route":
            case.update(bias=rng.random() < 0.5, groups=groups, top_groups=top_groups, group_score=rng.choice(["max", "top2"]),
                        align=rng.choice([1, 16]))
        return case
    if kind in ("gather", "combine", "combine_backward"):
        E = _log(rng, 4, 128)
        k = rng.randint(1, min(8, E))
        T, K = _log(rng, 1, 8192), _log(rng, 64, 8192, rng.choice([1, 8, 64]))
        T = max(1, min(T, MOST_VALUES // 2 // (k * K)))
        case = {"kind": kind, "t": rng.choice(["bf16", "bf16", "f16", "f32"] + (["e4m3", "i8"] if kind == "gather" else [])), "T": T, "K": K, "E": E,
                "k": k, "align": rng.choice([1, 16]), "dropped": rng.random() < 0.3}
        if case["t"] == "f32":
            case["T"] = max(1, T // 4)
        if kind == "combine":
            case.update(weights=rng.random() < 0.8, residual=rng.random() < 0.5)
        return case
    act = rng.choice(["", "relu", "gelu", "silu", "gelu_tanh"])
    if kind in ("linear", "linear_backward"):
        M, K, E = _log(rng, 64, 8192, 32), _log(rng, 64, 4096, 32), _log(rng, 1, 64)
        E = max(1, min(E, MOST_WEIGHTS // 2 // (M * K)))
        rows = max(1, min(_log(rng, 1, 16384), MOST_PRODUCT // 2 // (M * K)))
        skew = rng.choice([0.0, 0.3, 1.0, 2.0])
        if kind == "linear_backward":
            return {"kind": kind, "ab": rng.choice(["bf16", "f16"]), "E": E, "M": M, "K": K, "rows": max(16, rows // 32 * 16), "skew": skew, "act": act}
        ab = rng.choice(["bf16", "bf16", "f16", "e4m3", "i8"])
        return {"kind": kind, "ab": ab, "cd": ab if BYTES[ab] == 2 else rng.choice(["bf16", "f16"]), "E": E, "M": M, "K": K, "rows": rows,
                "skew": skew, "act": act, "bias": rng.random() < 0.6, "residual": rng.random() < 0.3, "pre": rng.random() < 0.3,
                "dense": rng.random() < 0.15}
    E = rng.choice([4, 8, 16, 32])
    K, F = _log(rng, 128, 2048, 32), _log(rng, 128, 1408, 32)
    case = {"kind": kind, "t": rng.choice(["bf16", "f16"]), "K": K, "F": F, "E": E, "k": rng.randint(1, 4), "act": rng.choice(["silu", "gelu"])}
    if kind == "layer":
        case.update(quant=rng.random() < 0.5, T=_log(rng, 1, 512))
    else:
        case.update(E=min(E, 8), T=_log(rng, 16, 2048))
    return case


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _normal(g, shape, sigma=1.0):
    return torch.randn(shape, generator=g, device="cuda") * sigma


def _row_scales(g, shape, size):
    return (torch.rand(shape, generator=g, device="cuda") + 0.5) * size


def _segments(case, unit):
    """How many rows each expert has: the same for every seed, more uneven with the skew, some experts without any."""
    rng = random.Random(f"{case['E']} {case['rows']} {case['skew']}")
    share = [math.exp(case["skew"] * rng.gauss(0, 1)) for _ in range(case["E"])]
    total, n, ends, run_ = sum(share), case["rows"] // unit, [0], 0.0
    for v in share:
        run_ += v
        ends.append(min(n, round(run_ / total * n)))
    ends[-1] = n
    return [e * unit for e in ends]


def _weights(g, E, M, K, ab):
    """Weights of E experts, M x K each, of which every aligned group of four along K has its two largest magnitudes."""
    out = torch.empty((E, M, K), dtype=DTYPE[ab], device="cuda")
    for e in range(E):
        w = _normal(g, (M, K), 1.0 / math.sqrt(K))
        if ab == "i8":
            w = (w * (32.0 * math.sqrt(K))).round().clamp_(-127, 127)
        elif ab == "e4m3":
            w = (w * (8.0 * math.sqrt(K))).to(DTYPE[ab]).float()
        else:
            w = w.to(DTYPE[ab]).float()
        a = w.abs().view(M, K // 4, 4).unbind(2)
        larger = [sum(((a[j] >= a[i]) if j < i else (a[j] > a[i])).to(torch.int8) for j in range(4) if j != i) for i in range(4)]
        keep = torch.stack([n < 2 for n in larger], 2)
        out[e] = (w * keep.view(M, K)).to(DTYPE[ab])
    return out


def _layer(g, E, M, K, ab, dense=False):
    """The experts' weights as a program keeps them: the pruned ones (training keeps them dense, as the plain form reads them)
    and, for the framework's products, their compressed form, laid out once."""
    layer = {"W": _weights(g, E, M, K, ab)}
    if own and not dense:
        from paper_2104_08378_b200 import binding as sp
        layer["vals"], layer["meta"] = sp.expert_compress(layer["W"])
    return layer


def _logits(g, T, E, t, masked):
    """Router logits; masked: experts that a token must not take, and tokens of a padded batch, are -inf."""
    logits = _normal(g, (T, E), 1.5)
    if masked:
        logits = logits.masked_fill(torch.rand((T, E), generator=g, device="cuda") < 0.2, -math.inf)
        logits[T - T // 8:] = -math.inf
    return logits.to(DTYPE[t])


def _choice(g, case):
    """k distinct experts of each token, popular ones more often; dropped: the last eighth of the tokens has none."""
    T, E = case["T"], case["E"]
    scores = _normal(g, (T, E)) + _normal(g, (E,), 0.7)
    experts = scores.topk(case["k"], dim=1).indices.to(torch.int32)
    if case["dropped"]:
        experts[T - T // 8:] = -1
    return experts


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case}
    kind = case["kind"]
    if kind in ("route", "route_backward"):
        T, E, t = case["T"], case["E"], case["t"]
        s["logits"] = _logits(g, T, E, t, case["masked"])
        if kind == "route":
            s["bias"] = _normal(g, (E,), 0.1 if case["score"] == "sigmoid" else 0.3 / E) if case["bias"] else None
        else:  # what the forward call has left: the experts that it chose
            s["experts"] = _route_plain(s["logits"], case["k"], case["score"])[1]
            s["dweights"] = _normal(g, (T, case["k"]))
    elif kind in ("gather", "combine", "combine_backward"):
        T, K, E, k, t = case["T"], case["K"], case["E"], case["k"], case["t"]
        experts = _choice(g, case)
        if own:
            from paper_2104_08378_b200 import binding as sp
            s["order"] = sp.expert_order(experts, E, align=case["align"])
            R = s["order"].source.shape[0]
        else:
            s["order"] = _order_plain(experts, E, case["align"])
            R = s["order"][2].shape[0]
        if kind == "gather":
            x = _normal(g, (T, K))
            s["x"] = (x * 32).round().clamp_(-127, 127).to(torch.int8) if t == "i8" else x.to(DTYPE[t])
            s["scale"] = _row_scales(g, (T,), 1.0 / 32) if BYTES[t] == 1 else None
        else:
            s["y"] = _normal(g, (R, K)).to(DTYPE[t])
            s["weights"] = _row_scales(g, (T, k), 1.0 / k) if case.get("weights", True) else None
            if kind == "combine":
                s["residual"] = _normal(g, (T, K)).to(DTYPE[t]) if case["residual"] else None
            else:
                s["dout"] = _normal(g, (T, K)).to(DTYPE[t])
    elif kind in ("linear", "linear_backward"):
        E, M, K, ab = case["E"], case["M"], case["K"], case["ab"]
        s["ends"] = _segments(case, 16 if kind == "linear_backward" else 1)  # (the plain form's: the host's copy)
        s["offsets"] = torch.tensor(s["ends"], dtype=torch.int32, device="cuda")
        R = s["ends"][-1]
        x = _normal(g, (R, K))
        s["X"] = (x * 32).round().clamp_(-127, 127).to(torch.int8) if ab == "i8" else x.to(DTYPE[ab])
        if kind == "linear":
            s.update(_layer(g, E, M, K, ab, case["dense"]))
            s["bias"] = _normal(g, (E, M), 0.5) if case["bias"] else None
            s["residual"] = _normal(g, (R, M)).to(DTYPE[case["cd"]]) if case["residual"] else None
            eight = BYTES[ab] == 1
            s["row_scale"] = _row_scales(g, (E, M), 1.0 / (32 * math.sqrt(K)) if ab == "i8" else 1.0 / (8 * math.sqrt(K))) if eight else None
            s["col_scale"] = _row_scales(g, (R,), 1.0 / 32 if ab == "i8" else 1.0) if eight else None
        else:
            s["W"] = _weights(g, E, M, K, ab)
            s["pre"] = _normal(g, (R, M)).to(DTYPE[ab])
            s["dy"] = _normal(g, (R, M)).to(DTYPE[ab])
    else:  # layer, layer_train
        T, K, F, E, t = case["T"], case["K"], case["F"], case["E"], case["t"]
        ab = "i8" if case.get("quant") else t
        s["x"] = _normal(g, (T, K)).to(DTYPE[t])
        s["logits"] = _logits(g, T, E, t, False)
        s["up"], s["down"] = _layer(g, E, 2 * F, K, ab), _layer(g, E, K, F, ab)
        if kind == "layer":
            s["weight"] = (_normal(g, (K,), 0.1) + 1.0).to(DTYPE[t])
            s["up_scale"] = _row_scales(g, (E, 2 * F), 1.0 / (32 * math.sqrt(K))) if ab == "i8" else None
            s["down_scale"] = _row_scales(g, (E, K), 1.0 / (32 * math.sqrt(F))) if ab == "i8" else None
        else:
            s["dout"] = _normal(g, (T, K)).to(DTYPE[t])
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2104_08378_b200 import binding as sp
    case = s["case"]
    kind = case["kind"]
    if kind == "route":
        weights, experts = sp.route(s["logits"], case["k"], score=case["score"], bias=s["bias"], groups=case["groups"], top_groups=case["top_groups"],
                                    group_score=case["group_score"], renorm=case["renorm"], scale=case["scale"])
        order = sp.expert_order(experts, case["E"], align=case["align"])
        return weights, experts, order.offsets, order.position, order.source
    if kind == "route_backward":
        return sp.route_backward(s["dweights"], s["logits"], s["experts"], score=case["score"], renorm=case["renorm"], scale=case["scale"])
    if kind == "gather":
        return sp.expert_gather(s["x"], s["order"], scale=s["scale"])
    if kind == "combine":
        return sp.expert_combine(s["y"], s["order"], s["weights"], residual=s["residual"])
    if kind == "combine_backward":
        return sp.expert_combine_backward(s["dout"], s["y"], s["order"], s["weights"])
    if kind == "linear":
        A, meta = (s["W"], None) if case["dense"] else (s["vals"], s["meta"])
        return sp.expert_linear(A, meta, s["X"], s["offsets"], bias=s["bias"], act=case["act"] or None, residual=s["residual"],
                                row_scale=s["row_scale"], col_scale=s["col_scale"], pre=case["pre"], cd=case["cd"], a_is_dense=case["dense"])
    if kind == "linear_backward":
        return sp.expert_linear_backward(s["dy"], s["pre"], s["X"], s["W"], s["offsets"], act=case["act"] or None)
    F, E, k, t, act = case["F"], case["E"], case["k"], case["t"], case["act"]
    if kind == "layer":
        q = "i8" if case["quant"] else None
        weights, experts = sp.route(s["logits"], k)
        order = sp.expert_order(experts, E)
        h, _, scale, _ = sp.rms_norm(s["x"], s["weight"], eps=EPS, quant=q)
        hs, scales = sp.expert_gather(h, order, scale=scale)
        gu = sp.expert_linear(s["up"]["vals"], s["up"]["meta"], hs, order.offsets, row_scale=s["up_scale"], col_scale=scales, cd=t)
        a, a_scale = sp.gated_act(gu[:, :F], gu[:, F:], act=act, quant=q)
        y = sp.expert_linear(s["down"]["vals"], s["down"]["meta"], a, order.offsets, row_scale=s["down_scale"], col_scale=a_scale, cd=t)
        return sp.expert_combine(y, order, weights, residual=s["x"])
    weights, experts = sp.route(s["logits"], k)
    order = sp.expert_order(experts, E, align=16)
    xs, _ = sp.expert_gather(s["x"], order)
    gu = sp.expert_linear(s["up"]["vals"], s["up"]["meta"], xs, order.offsets)
    a, _ = sp.gated_act(gu[:, :F], gu[:, F:], act=act)
    y = sp.expert_linear(s["down"]["vals"], s["down"]["meta"], a, order.offsets)
    out = sp.expert_combine(y, order, weights, residual=s["x"])
    dy, dweights = sp.expert_combine_backward(s["dout"], y, order, weights)
    da, d_down, _ = sp.expert_linear_backward(dy, None, a, s["down"]["W"], order.offsets, meta=s["down"]["meta"], bias=False)
    dgu = torch.empty_like(gu)
    sp.gated_act_backward(da, gu[:, :F], gu[:, F:], act=act, dg=dgu[:, :F], du=dgu[:, F:])
    dxs, d_up, _ = sp.expert_linear_backward(dgu, None, xs, s["up"]["W"], order.offsets, meta=s["up"]["meta"], bias=False)
    dx = sp.expert_combine(dxs, order, residual=s["dout"])
    return out, dx, d_up, d_down, sp.route_backward(dweights, s["logits"], experts)


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


def _best(v, k):
    """The k largest of each row and their indices, the lower index first among equal ones."""
    order = torch.sort(v, dim=1, descending=True, stable=True)
    return order.values[:, :k], order.indices[:, :k]


def _scores(logits, score):
    if score == "sigmoid":
        return 1 / (1 + torch.exp(-logits))
    top = logits.amax(1, keepdim=True)
    p = torch.exp(logits - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    return p / p.sum(1, keepdim=True).clamp(min=1e-300 if logits.dtype == torch.float64 else 1e-37)


def _route_plain(logits, k, score="softmax", bias=None, groups=1, top_groups=1, group_score="max", renorm=True, scale=1.0):
    T, E = logits.shape
    l = logits.float()
    d = l.double()
    # what an expert is chosen by: next to a border 32 bits would not do
    choose = d if bias is None else torch.where(d > -math.inf, _scores(d, score) + bias.double(), d)
    if groups > 1:
        by = choose
        if group_score == "top2" and bias is None:
            by = torch.where(d > -math.inf, _scores(d, score), d)
        best, _ = _best(by.reshape(T * groups, E // groups), 2 if group_score == "top2" and E // groups > 1 else 1)
        group = torch.where(best > -math.inf, best, torch.zeros_like(best)).sum(1)
        group = torch.where(best[:, 0] > -math.inf, group, best[:, 0]).view(T, groups)
        chosen = torch.zeros((T, groups), dtype=torch.bool, device=l.device).scatter_(1, _best(group, top_groups)[1], True)
        choose = torch.where(chosen[:, :, None].expand(T, groups, E // groups).reshape(T, E), choose, torch.full_like(choose, -math.inf))
    value, experts = _best(choose, k)
    live = value > -math.inf
    s = torch.where(live, torch.gather(_scores(l, score), 1, experts), torch.zeros_like(value, dtype=torch.float32))
    if renorm:
        s = s / s.sum(1, keepdim=True).clamp(min=1e-37)
    return s * scale, torch.where(live, experts, torch.full_like(experts, -1)).to(torch.int32)


def _order_plain(experts, E, align):
    """(offsets, position, source): the first row of each expert, the row of each token's slot (-1: none), and the slot (token
    * k + number) of each row (-1: none)."""
    T, k = experts.shape
    n = T * k
    flat = experts.reshape(-1).long()
    slot = torch.arange(n, device=flat.device)
    key = torch.where(flat < 0, torch.full_like(flat, E), flat)
    by = torch.sort(key, stable=True)
    counts = torch.zeros(E + 1, dtype=torch.long, device=flat.device).index_add_(0, key, torch.ones_like(key))[:E]
    padded = (counts + align - 1) // align * align
    offsets = torch.zeros(E + 1, dtype=torch.long, device=flat.device)
    offsets[1:] = padded.cumsum(0)
    first = torch.zeros(E + 1, dtype=torch.long, device=flat.device)
    first[1:] = counts.cumsum(0)
    place = slot - first[by.values] + offsets[by.values]  # of the sorted slots
    R = (n + (align - 1) * min(E, n) + align - 1) // align * align
    dead = by.values == E
    position = torch.full((n,), -1, dtype=torch.int32, device=flat.device)
    position[by.indices] = torch.where(dead, torch.full_like(place, -1), place).to(torch.int32)
    source = torch.full((R + 1,), -1, dtype=torch.int32, device=flat.device)
    source[torch.where(dead, torch.full_like(place, R), place)] = by.indices.to(torch.int32)
    return offsets.to(torch.int32), position.view(T, k), source[:R]  # (slots without a row went behind the end)


def _rows_at(y, position):
    """Rows of y at positions of any shape; zeros where there is none."""
    rows = y[position.clamp(min=0).long()]
    return torch.where((position >= 0)[..., None], rows, torch.zeros_like(rows))


def _quantised(y):
    scale = y.abs().amax(1) / 127.0
    q = y / torch.where(scale > 0, scale, torch.ones_like(scale))[:, None]
    return q.round().to(torch.int8), scale


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "route":
        weights, experts = _route_plain(s["logits"], case["k"], case["score"], s["bias"], case["groups"], case["top_groups"], case["group_score"],
                                        case["renorm"], case["scale"])
        return (weights, experts) + _order_plain(experts, case["E"], case["align"])
    if kind == "route_backward":
        return _route_backward_plain(s["dweights"], s["logits"], s["experts"], case["score"], case["renorm"], case["scale"])
    if kind == "gather":
        token = torch.where(s["order"][2] >= 0, s["order"][2] // case["k"], s["order"][2])
        scale = None if s["scale"] is None else _rows_at(s["scale"][:, None], token)[:, 0]
        if BYTES[case["t"]] == 1:
            return _rows_at(s["x"].view(torch.int8), token).view(s["x"].dtype), scale
        return _rows_at(s["x"], token), scale
    if kind == "combine":
        rows = _rows_at(s["y"], s["order"][1]).float()
        out = (rows if s["weights"] is None else rows * s["weights"][:, :, None]).sum(1)
        return (out if s["residual"] is None else out + s["residual"].float()).to(s["y"].dtype)
    if kind == "combine_backward":
        _, position, source = s["order"]
        dw = (_rows_at(s["y"], position).float() * s["dout"].float()[:, None, :]).sum(2)
        w = torch.where(source >= 0, s["weights"].reshape(-1)[source.clamp(min=0).long()], torch.zeros((), device="cuda"))
        dy = s["dout"][(source.clamp(min=0) // case["k"]).long()].float() * w[:, None]
        return dy.to(s["y"].dtype), dw
    if kind == "linear":
        ends, ys, zs = s["ends"], [], []
        for e in range(case["E"]):
            lo, hi = ends[e], ends[e + 1]
            if lo == hi:
                continue
            z = s["X"][lo:hi].float() @ s["W"][e].float().T
            if s["row_scale"] is not None:
                z = z * s["col_scale"][lo:hi, None] * s["row_scale"][e][None, :]
            if s["bias"] is not None:
                z = z + s["bias"][e]
            y = _act(z, case["act"])
            if s["residual"] is not None:
                y = y + s["residual"][lo:hi].float()
            ys.append(y.to(DTYPE[case["cd"]]))
            zs.append(z.to(DTYPE[case["cd"]]))
        return (torch.cat(ys), torch.cat(zs)) if case["pre"] else torch.cat(ys)
    if kind == "linear_backward":
        ends, dXs, dWs, dbs = s["ends"], [], [], []
        for e in range(case["E"]):
            lo, hi = ends[e], ends[e + 1]
            dz = s["dy"][lo:hi].float() * _act_slope(s["pre"][lo:hi].float(), case["act"])
            dXs.append((dz @ s["W"][e].float()).to(s["W"].dtype))
            dWs.append((dz.T @ s["X"][lo:hi].float()).to(s["W"].dtype))
            dbs.append(dz.sum(0))
        return torch.cat(dXs), torch.stack(dWs), torch.stack(dbs)
    F, E, t, act, x = case["F"], case["E"], DTYPE[case["t"]], case["act"], s["x"]
    weights, experts = _route_plain(s["logits"], case["k"])
    if kind == "layer":
        f = x.float()
        h = f * (f.square().mean(1, keepdim=True) + EPS).rsqrt() * s["weight"].float()
        h, h_scale = _quantised(h) if case["quant"] else (h.to(t), None)
    else:
        h, h_scale = x, None
    T, K = x.shape
    ys = torch.zeros((T, case["k"], K), dtype=t, device="cuda")
    kept = []
    for e in range(E):  # every expert over all tokens; what a token did not choose is left out
        chosen = experts == e
        gu = h.float() @ s["up"]["W"][e].float().T
        if h_scale is not None:
            gu = gu * h_scale[:, None] * s["up_scale"][e]
        gu = gu.to(t).float()
        a = _act(gu[:, :F], act) * gu[:, F:]
        if h_scale is not None:
            a, a_scale = _quantised(a)
            y = (a.float() @ s["down"]["W"][e].float().T) * a_scale[:, None] * s["down_scale"][e]
        else:
            a = a.to(t)
            y = a.float() @ s["down"]["W"][e].float().T
        ys = torch.where(chosen[:, :, None], y.to(t)[:, None, :], ys)
        if kind == "layer_train":
            kept.append((chosen, gu, a))
    out = ((ys.float() * weights[:, :, None]).sum(1) + x.float()).to(t)
    if kind == "layer":
        return out
    dout = s["dout"].float()
    dweights = (ys.float() * dout[:, None, :]).sum(2)
    dx, d_up, d_down = torch.zeros((T, K), device="cuda"), [], []
    for e, (chosen, gu, a) in enumerate(kept):
        dy = (dout * torch.where(chosen, weights, torch.zeros_like(weights)).sum(1, keepdim=True)).to(t).float()
        Wd, Wu = s["down"]["W"][e], s["up"]["W"][e]
        da = (dy @ Wd.float()).to(t).float()
        d_down.append(torch.where(Wd != 0, dy.T @ a.float(), torch.zeros((), device="cuda")).to(t))
        dgu = torch.cat([da * gu[:, F:] * _act_slope(gu[:, :F], act), da * _act(gu[:, :F], act)], 1).to(t).float()
        d_up.append(torch.where(Wu != 0, dgu.T @ x.float(), torch.zeros((), device="cuda")).to(t))
        dx = dx + (dgu @ Wu.float()).to(t).float()
    return out, (dx + dout).to(t), torch.stack(d_up), torch.stack(d_down), _route_backward_plain(dweights, s["logits"], experts)


def _route_backward_plain(dweights, logits, experts, score="softmax", renorm=True, scale=1.0):
    l = logits.float()
    live = experts >= 0
    at = experts.clamp(min=0).long()
    g = torch.where(live, dweights * scale, torch.zeros_like(dweights))
    p = torch.where(live, torch.gather(_scores(l, score), 1, at), torch.zeros_like(g))
    if renorm:
        u = p / p.sum(1, keepdim=True).clamp(min=1e-37)
        dz = u * (g - (u * g).sum(1, keepdim=True))  # of the logarithm of the chosen experts' scores
        dz = torch.where(live, dz * (1 - p) if score == "sigmoid" else dz, torch.zeros_like(dz))
        return torch.zeros_like(l).scatter_add_(1, at, dz).to(logits.dtype)
    if score == "sigmoid":
        return torch.zeros_like(l).scatter_add_(1, at, g * p * (1 - p)).to(logits.dtype)
    full = torch.zeros_like(l).scatter_add_(1, at, g)
    return (_scores(l, score) * (full - (p * g).sum(1, keepdim=True))).to(logits.dtype)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------
def _weight_bytes(M, K, ab, dense=False):
    """Compressed weights: half the values and two bits for each."""
    return M * K * BYTES[ab] if dense else M * K // 2 * BYTES[ab] + M * K // 8


def _rows(case):
    return (case["T"] - (case["T"] // 8 if case["dropped"] else 0)) * case["k"]


def _experts_met(case):
    """Experts that T tokens with k of E each can be expected to meet."""
    return max(min(case["E"], case["k"]), round(case["E"] * (1 - (1 - min(1.0, case["k"] / case["E"])) ** case["T"])))


def work(case):
    kind = case["kind"]
    if kind in ("route", "route_backward"):
        T, E, k, e = case["T"], case["E"], case["k"], BYTES[case["t"]]
        if kind == "route":
            return {"bytes": T * E * e + 4 * T * k * 4 + 4 * (E + 1), "flops": 4 * T * E}
        return {"bytes": 2 * T * E * e + 2 * 4 * T * k, "flops": 4 * T * E}
    if kind in ("gather", "combine", "combine_backward"):
        T, K, k, e, R = case["T"], case["K"], case["k"], BYTES[case["t"]], _rows(case)
        if kind == "gather":
            return {"bytes": (T + R) * (K * e + (4 if e == 1 else 0)) + 4 * R, "flops": 0}
        if kind == "combine":
            return {"bytes": (R + T * (2 if case["residual"] else 1)) * K * e + 4 * T * k * (2 if case["weights"] else 1), "flops": 2 * R * K}
        return {"bytes": (T + 2 * R) * K * e + 4 * T * k * 3, "flops": 3 * R * K}
    if kind in ("linear", "linear_backward"):
        M, K, e = case["M"], case["K"], BYTES[case["ab"]]
        ends = _segments(case, 16 if kind == "linear_backward" else 1)
        R, met = ends[-1], sum(1 for a, b in zip(ends, ends[1:]) if b > a)
        if kind == "linear":
            c, outs = BYTES[case["cd"]], 1 + bool(case["residual"]) + bool(case["pre"])
            vectors = 4 * met * M * (bool(case["bias"]) + (e == 1)) + (4 * R if e == 1 else 0)
            return {"bytes": met * _weight_bytes(M, K, case["ab"], case["dense"]) + R * K * e + outs * R * M * c + vectors,
                    "flops": R * M * K * (2 if case["dense"] else 1)}  # half of the sparse weights are zeros
        act = 2 if case["act"] else 1
        return {"bytes": e * (act * R * M + 2 * R * K + met * M * K + case["E"] * M * K) + 4 * case["E"] * M, "flops": 4 * R * M * K}
    T, K, F, E, k, e = case["T"], case["K"], case["F"], case["E"], case["k"], BYTES[case["t"]]
    met, R = _experts_met(case), T * k
    if kind == "layer":
        ab = "i8" if case["quant"] else case["t"]
        vectors = 4 * met * (2 * F + K) if case["quant"] else 0
        return {"bytes": met * (_weight_bytes(2 * F, K, ab) + _weight_bytes(K, F, ab)) + vectors + 2 * T * K * e + T * E * e, "flops": 3 * R * K * F}
    sparse = met * (_weight_bytes(2 * F, K, case["t"]) + _weight_bytes(K, F, case["t"]))
    return {"bytes": sparse + e * (met * 3 * F * K + E * 3 * F * K + 4 * T * K + 2 * T * E), "flops": 3 * R * K * F + 12 * R * K * F}


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


def _route64(logits, k, score="softmax", bias=None, groups=1, top_groups=1, group_score="max", renorm=True, scale=1.0):
    """Expert after expert: the best of those that are left, the first of equal ones."""
    T, E = logits.shape
    l = logits.double()
    none = torch.isneginf(l)
    s = torch.sigmoid(l) if score == "sigmoid" else torch.softmax(l, 1).nan_to_num(0.0)  # (nothing to choose from: no score)
    left = l.clone() if bias is None else (s + bias.double()).masked_fill(none, -math.inf)
    rows = torch.arange(T, device=l.device)
    if groups > 1:
        n = E // groups
        by = (s.masked_fill(none, -math.inf) if bias is None and group_score == "top2" else left).view(T, groups, n)
        value = by.amax(2)
        if group_score == "top2" and n > 1:
            second = by.clone().scatter_(2, by.argmax(2, keepdim=True), -math.inf).amax(2)
            value = value + torch.where(torch.isneginf(second), torch.zeros_like(second), second)
        open_ = torch.zeros((T, groups), dtype=torch.bool, device=l.device)
        for _ in range(top_groups):
            first = ((value == value.amax(1, keepdim=True)) & ~open_).to(torch.int8).argmax(1)
            open_[rows, first] = True
            value[rows, first] = -math.inf
        left = left.masked_fill(~open_.repeat_interleave(n, 1), -math.inf)
    experts, weights = [], []
    for _ in range(k):
        top = left.amax(1)
        first = (left == top[:, None]).to(torch.int8).argmax(1)
        dead = torch.isneginf(top)
        experts.append(torch.where(dead, torch.full_like(first, -1), first))
        weights.append(torch.where(dead, torch.zeros_like(top), s[rows, first]))
        left[rows, first] = -math.inf
    w = torch.stack(weights, 1)
    if renorm:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    return w * scale, torch.stack(experts, 1).to(torch.int32)


def _order64(experts, E, align):
    """Row after row, on the host."""
    T, k = experts.shape
    lists = [[] for _ in range(E)]
    for i, e in enumerate(experts.reshape(-1).tolist()):
        if e >= 0:
            lists[e].append(i)
    n = T * k
    R = -(-(n + (align - 1) * min(E, n)) // align) * align
    offsets, position, source = [0], [-1] * n, [-1] * R
    for slots in lists:
        for j, i in enumerate(slots):
            position[i], source[offsets[-1] + j] = offsets[-1] + j, i
        offsets.append(offsets[-1] + -(-len(slots) // align) * align)
    dev = experts.device
    return (torch.tensor(offsets, dtype=torch.int32, device=dev), torch.tensor(position, dtype=torch.int32, device=dev).view(T, k),
            torch.tensor(source, dtype=torch.int32, device=dev))


def _route_backward64(dweights, logits, experts, score="softmax", renorm=True, scale=1.0):
    """By the Jacobian of the chosen experts' weights: dw_s / dl_e."""
    T, E = logits.shape
    l = logits.double()
    live = experts >= 0
    pick = torch.zeros((T, experts.shape[1], E), dtype=torch.float64, device=l.device)
    pick.scatter_(2, experts.clamp(min=0).long()[:, :, None], 1.0)
    pick = pick * live[:, :, None]
    s = torch.sigmoid(l) if score == "sigmoid" else torch.softmax(l, 1).nan_to_num(0.0)
    g = dweights.double().masked_fill(~live, 0.0) * scale
    ps = torch.einsum("tse,te->ts", pick, s)
    if renorm:  # w_s = p_s / sum p
        total = ps.sum(1, keepdim=True).clamp(min=1e-300)
        g = g / total - (g * ps).sum(1, keepdim=True) / total ** 2
    ds = torch.einsum("tse,ts->te", pick, g)  # with respect to the scores
    if score == "sigmoid":
        return ds * s * torch.sigmoid(-l)
    return s * (ds - (s * ds).sum(1, keepdim=True))


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "route":
        weights, experts = _route64(s["logits"], case["k"], case["score"], s["bias"], case["groups"], case["top_groups"], case["group_score"],
                                    case["renorm"], case["scale"])
        return (weights, experts) + _order64(experts, case["E"], case["align"])
    if kind == "route_backward":
        if case["T"] * case["k"] * case["E"] > 1 << 28:
            parts = [slice(i, i + 4096) for i in range(0, case["T"], 4096)]
            return torch.cat([_route_backward64(s["dweights"][p], s["logits"][p], s["experts"][p], case["score"], case["renorm"], case["scale"]) for p in parts])
        return _route_backward64(s["dweights"], s["logits"], s["experts"], case["score"], case["renorm"], case["scale"])
    if kind in ("gather", "combine", "combine_backward"):
        position, source = (s["order"].position, s["order"].source) if own else s["order"][1:]
        token = torch.div(source.clamp(min=0), case["k"], rounding_mode="floor").long()
        used = (source >= 0)[:, None]
        if kind == "gather":
            return s["x"].double()[token] * used, None if s["scale"] is None else s["scale"].double()[token] * used[:, 0]
        y, w = s["y"].double(), s["weights"]
        w = torch.ones(position.shape, dtype=torch.float64, device="cuda") if w is None else w.double()
        if kind == "combine":
            out = torch.zeros((case["T"], case["K"]), dtype=torch.float64, device="cuda")
            out.index_add_(0, token, y * (used * w.reshape(-1)[source.clamp(min=0).long()][:, None]))  # row after row to its token
            return out if s["residual"] is None else out + s["residual"].double()
        dout = s["dout"].double()[token] * used
        dw = torch.zeros(position.numel(), dtype=torch.float64, device="cuda")
        dw.index_add_(0, source.clamp(min=0).long(), torch.einsum("rk,rk->r", dout, y))
        return dout * w.reshape(-1)[source.clamp(min=0).long()][:, None], dw.view(position.shape)
    if kind in ("linear", "linear_backward"):
        ends, outs = s["ends"], []
        for e in range(case["E"]):
            rows = slice(ends[e], ends[e + 1])
            x, W = s["X"][rows].double(), s["W"][e].double()
            if kind == "linear":
                z = torch.einsum("rk,mk->rm", x, W)
                if s["row_scale"] is not None:
                    z = z * torch.outer(s["col_scale"][rows].double(), s["row_scale"][e].double())
                z = z if s["bias"] is None else z + s["bias"][e].double()[None, :]
                y = _act64(z, case["act"])[0]
                outs.append((y if s["residual"] is None else y + s["residual"][rows].double(), z))
            else:
                dz = s["dy"][rows].double() * _act64(s["pre"][rows].double(), case["act"])[1]
                outs.append((torch.einsum("rm,mk->rk", dz, W), torch.einsum("rm,rk->mk", dz, x), dz.sum(0)))
        if kind == "linear_backward":
            return torch.cat([o[0] for o in outs]), torch.stack([o[1] for o in outs]), torch.stack([o[2] for o in outs])
        y = torch.cat([o[0] for o in outs])
        return (y, torch.cat([o[1] for o in outs])) if case["pre"] else y
    # the layers: expert after expert over the rows that chose it, intermediate results held in the types that the definition names
    F, E, act, x, t = case["F"], case["E"], case["act"], s["x"], s["x"].dtype
    weights, experts = _route64(s["logits"], case["k"])
    held = lambda v: v.to(t).double()  # noqa: E731
    h = x.double()
    scale = None
    if kind == "layer":
        h = s["weight"].double()[None, :] * h / torch.sqrt((h * h).sum(1, keepdim=True) / h.shape[1] + EPS)
        if case["quant"]:
            scale = h.abs().amax(1) / 127.0
            h = torch.round(h / scale.clamp(min=1e-300)[:, None])
        else:
            h = held(h)
    out, met = x.double().clone(), []
    for e in range(E):
        token, slot = (experts == e).nonzero(as_tuple=True)
        Wu, Wd = s["up"]["W"][e].double(), s["down"]["W"][e].double()
        gu = h[token] @ Wu.T
        if scale is not None:
            gu = gu * torch.outer(scale[token], s["up_scale"][e].double())
        gu = held(gu)
        a = _act64(gu[:, :F], act)[0] * gu[:, F:]
        if scale is not None:
            a_scale = a.abs().amax(1) / 127.0
            y = torch.round(a / a_scale.clamp(min=1e-300)[:, None]) @ Wd.T * torch.outer(a_scale, s["down_scale"][e].double())
        else:
            a = held(a)
            y = a @ Wd.T
        y = held(y)
        out.index_add_(0, token, y * weights[token, slot][:, None])
        met.append((token, slot, gu, a, y))
    if kind == "layer":
        return out
    dx, d_up, d_down = s["dout"].double().clone(), [], []
    dweights = torch.zeros(experts.shape, dtype=torch.float64, device="cuda")
    for e, (token, slot, gu, a, y) in enumerate(met):
        Wu, Wd = s["up"]["W"][e].double(), s["down"]["W"][e].double()
        d = s["dout"].double()[token]
        dweights[token, slot] = (d * y).sum(1)
        dy = held(d * weights[token, slot][:, None])
        da = held(dy @ Wd)
        value, slope = _act64(gu[:, :F], act)
        dgu = held(torch.cat([da * gu[:, F:] * slope, da * value], 1))
        d_down.append((dy.T @ a) * (Wd != 0))
        d_up.append((dgu.T @ x.double()[token]) * (Wu != 0))
        dx.index_add_(0, token, held(dgu @ Wu))
    return out, dx, torch.stack(d_up), torch.stack(d_down), _route_backward64(dweights, s["logits"], experts)
