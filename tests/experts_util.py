"""What the tests of the experts' operators share: plain implementations, token after token and row after row."""
import math

import torch


def route64(logits, k, score="softmax", bias=None, groups=1, top_groups=None, group_score="max", renorm=True, scale=1.0):
    """(weights, experts) in 64 bits on the host, with Python's sort: by value, then by index."""
    top_groups = groups if top_groups is None else top_groups
    T, E = logits.shape
    n = E // groups
    weights, experts = torch.zeros((T, k), dtype=torch.float64), torch.full((T, k), -1, dtype=torch.int32)
    s_all = torch.sigmoid(logits.double()) if score == "sigmoid" else torch.softmax(logits.double(), 1)
    l_all, s_all = logits.double().cpu().tolist(), s_all.cpu().tolist()
    b = None if bias is None else bias.double().cpu().tolist()
    for t in range(T):
        l, s = l_all[t], s_all[t]
        live = [e for e in range(E) if l[e] > -math.inf and (b is None or b[e] > -math.inf)]
        by = {e: l[e] if b is None else s[e] + b[e] for e in live}
        if groups > 1:
            value = {}
            for g in range(groups):
                if group_score == "top2" and n > 1:
                    best = sorted((s[e] + (b[e] if b else 0.0) for e in live if e // n == g), reverse=True)[:2]
                    if best:
                        value[g] = sum(best)
                else:
                    best = [by[e] for e in live if e // n == g]
                    if best:
                        value[g] = max(best)
            kept = sorted(value, key=lambda g: (-value[g], g))[:top_groups]
            live = [e for e in live if e // n in kept]
        chosen = sorted(live, key=lambda e: (-by[e], e))[:k]
        if renorm:  # in proportion to the scores, by their logarithms
            z = [l[e] if score == "softmax" else -math.log1p(math.exp(-l[e])) if l[e] > -700 else l[e] for e in chosen]
            w = [math.exp(v - max(z)) for v in z]
            w = [scale * v / sum(w) for v in w]
        else:
            w = [scale * s[e] for e in chosen]
        for i, e in enumerate(chosen):
            experts[t, i], weights[t, i] = e, w[i]
    return weights.to(logits.device), experts.to(logits.device)


def order_of(experts, E, align):
    """(offsets, position, source) slot after slot, on the host."""
    T, k = experts.shape
    slots = [[] for _ in range(E)]
    for i, e in enumerate(experts.reshape(-1).tolist()):
        if 0 <= e < E:
            slots[e].append(i)
    n = T * k
    rows = -(-(n + (align - 1) * min(E, n)) // align) * align
    offsets, position, source = [0], [-1] * n, [-1] * rows
    for mine in slots:
        for j, i in enumerate(mine):
            position[i], source[offsets[-1] + j] = offsets[-1] + j, i
        offsets.append(offsets[-1] + -(-len(mine) // align) * align)
    return torch.tensor(offsets, dtype=torch.int32), torch.tensor(position, dtype=torch.int32).view(T, k), torch.tensor(source, dtype=torch.int32)


def choice(T, E, k, seed, dropped=0.0):
    """k distinct experts of each token, some slots of it dropped."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    experts = torch.rand((T, E), generator=g, device="cuda").topk(k, dim=1).indices.to(torch.int32)
    return experts.masked_fill(torch.rand((T, k), generator=g, device="cuda") < dropped, -1)
