"""What routing to experts and low-rank adapters are timed on, and their plain forms.

Operators: the choice of experts for every token (softmax or sigmoid scores, a bias for balance, groups, top k,
renormalised weights); the sort of the chosen (token, expert) pairs by expert that products over groups of rows need; the
weighted sum of the experts' result rows back at their tokens; and a projection with low-rank adapters beside it, one or
several per row, as a batch of requests or a router picks them.  Sizes are those of the repository's blocks (width 3072,
QKV of 9216, MLP of 12288, 820 edited rows, 8704 rows of a full forward) and of generic expert layers.
"""
from __future__ import annotations

import math
import random

import torch

own = False


# ------------------------------------------------------------------------------------------------ the cases


def listed():
    return [
        # One token of a small expert layer: launch latency.
        {"name": "route_1_token", "op": "route", "tokens": 1, "experts": 64, "score": "softmax", "dtype": "f32", "bias": False, "groups": 1, "top_groups": 1,
         "best": 1, "k": 6, "renorm": True, "scale": 1.0, "masked": 0.0},
        # Text and image tokens of a 64x64 image, sigmoid scores with a balancing bias, the best four of eight groups.
        {"name": "route_4608_tokens_groups", "op": "route", "tokens": 4608, "experts": 256, "score": "sigmoid", "dtype": "f32", "bias": True, "groups": 8,
         "top_groups": 4, "best": 2, "k": 8, "renorm": True, "scale": 2.5, "masked": 0.0},
        # A large batch, scores in bf16 (many ties), an eighth of the tokens is padding.
        {"name": "route_65536_tokens", "op": "route", "tokens": 65536, "experts": 128, "score": "softmax", "dtype": "bf16", "bias": False, "groups": 1,
         "top_groups": 1, "best": 1, "k": 8, "renorm": True, "scale": 1.0, "masked": 0.125},
        # 36 edited tokens, two of 16 experts each: launch latency.
        {"name": "slots_36_tokens", "op": "slots", "tokens": 36, "experts": 16, "k": 2, "masked": 0.0, "spread": "even"},
        # The same large batch behind the router, experts of very different popularity.
        {"name": "slots_65536_tokens", "op": "slots", "tokens": 65536, "experts": 128, "k": 8, "masked": 0.125, "spread": "skewed"},
        # Eight tokens of the residual stream, float32.
        {"name": "combine_8_tokens", "op": "combine", "tokens": 8, "k": 2, "cols": 3072, "dtype": "f32", "out": "f32", "base": True, "masked": 0.0},
        # An expert layer's results on many tokens: HBM.
        {"name": "combine_16384_tokens", "op": "combine", "tokens": 16384, "k": 4, "cols": 4096, "dtype": "bf16", "out": "bf16", "base": True, "masked": 0.0},
        # One edited token through a QKV projection with its request's adapter: the weights from HBM.
        {"name": "adapters_1_row_qkv", "op": "adapters", "m": 1, "n": 9216, "k": 3072, "rank": 16, "adapters": 4, "sel": 1, "who": "requests", "requests": 1,
         "act": "none", "out": "bf16", "bias": True},
        # 48 requests of one row each, most with an adapter of their own.
        {"name": "adapters_48_requests", "op": "adapters", "m": 48, "n": 4096, "k": 2048, "rank": 16, "adapters": 32, "sel": 1, "who": "requests", "requests": 48,
         "act": "none", "out": "bf16", "bias": False},
        # MLP up of the benchmark block, 20 % of a 64x64 image edited: five requests, two weighted adapters each.
        {"name": "adapters_820_rows_mlp_up", "op": "adapters", "m": 820, "n": 12288, "k": 3072, "rank": 32, "adapters": 6, "sel": 2, "who": "requests", "requests": 5,
         "act": "gelu", "out": "bf16", "bias": True},
        # A mixture of low-rank experts: every token has two of eight, float32 result.
        {"name": "adapters_4096_tokens_mixture", "op": "adapters", "m": 4096, "n": 2048, "k": 2048, "rank": 16, "adapters": 8, "sel": 2, "who": "router", "requests": 1,
         "act": "none", "out": "f32", "bias": True},
        # QKV of a full forward, four requests with an adapter each.
        {"name": "adapters_8704_rows_qkv", "op": "adapters", "m": 8704, "n": 9216, "k": 3072, "rank": 64, "adapters": 4, "sel": 1, "who": "requests", "requests": 4,
         "act": "none", "out": "bf16", "bias": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["route", "route", "slots", "combine", "adapters", "adapters", "adapters"])
    masked = rng.choice([0.0, 0.0, 0.1, 0.5])
    if op == "route":
        groups = rng.choice([1, 1, 4, 8])
        experts = groups * _log_int(rng, 4, 32) if groups > 1 else _log_int(rng, 8, 256)
        top_groups = rng.randint(1, groups)
        k = min(_log_int(rng, 1, 10), top_groups * (experts // groups))
        return {"op": op, "tokens": _log_int(rng, 1, 65536 * 128 // max(128, experts)), "experts": experts, "score": rng.choice(["softmax", "sigmoid"]),
                "dtype": rng.choice(["f32", "bf16"]), "bias": rng.random() < 0.5, "groups": groups, "top_groups": top_groups, "best": rng.choice([1, 2]), "k": k,
                "renorm": rng.random() < 0.7, "scale": rng.choice([1.0, 2.5]), "masked": masked}
    if op == "slots":
        experts = _log_int(rng, 4, 256)
        return {"op": op, "tokens": _log_int(rng, 1, 65536), "experts": experts, "k": min(_log_int(rng, 1, 8), experts), "masked": masked,
                "spread": rng.choice(["even", "skewed", "one"])}
    if op == "combine":
        k, cols = _log_int(rng, 1, 8), _log_int(rng, 64, 4096) if rng.random() < 0.3 else 8 * _log_int(rng, 8, 512)
        return {"op": op, "tokens": _log_int(rng, 1, 16384 * 4 // max(4, k)), "k": k, "cols": cols, "dtype": rng.choice(["bf16", "f32"]), "out": rng.choice(["bf16", "f32"]),
                "base": rng.random() < 0.5, "masked": masked}
    m = _log_int(rng, 1, 8704)
    n = _log_int(rng, 64, 9216) if rng.random() < 0.3 else 8 * _log_int(rng, 16, 1152)
    k = 64 * _log_int(rng, 2, 192 if m < 1000 else 48)
    rank = _log_int(rng, 4, 64)
    adapters = _log_int(rng, 1, max(2, min(64, 512 // rank)))
    who = rng.choice(["requests", "requests", "router"])
    sel = min(adapters, rng.choice([1, 1, 2, 3]))
    return {"op": op, "m": m, "n": n, "k": k, "rank": rank, "adapters": adapters, "sel": sel, "who": who, "requests": _log_int(rng, 1, min(m, 64)),
            "act": rng.choice(["none", "gelu"]), "out": rng.choice(["bf16", "bf16", "f32"]), "bias": rng.random() < 0.8}


# ------------------------------------------------------------------------------------------------ inputs


_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _route_inputs(case, seed):
    """Scores of a router: a common preference of the experts, and the tokens' own; a bias that works against the preference."""
    g = _generator(seed)
    n, e = case["tokens"], case["experts"]
    liked = 0.7 * torch.randn(e, generator=g, device="cuda")
    logits = (liked + 1.2 * torch.randn((n, e), generator=g, device="cuda")).to(_TYPES[case["dtype"]])
    bias = -0.1 * liked + 0.02 * torch.randn(e, generator=g, device="cuda") if case["bias"] else None
    mask = (torch.rand(n, generator=g, device="cuda") >= case["masked"]).to(torch.uint8) if case["masked"] > 0 else None
    return logits, bias, mask


def _slots_inputs(case, seed):
    """What a router hands on: distinct experts per token, -1 for tokens that are not routed."""
    g = _generator(seed)
    n, e, k = case["tokens"], case["experts"], case["k"]
    liked = {"even": 0.0, "skewed": 1.5, "one": 40.0}[case["spread"]] * torch.randn(e, generator=g, device="cuda")
    expert = (liked + torch.randn((n, e), generator=g, device="cuda")).topk(k, dim=1).indices.to(torch.int32)
    expert[torch.rand(n, generator=g, device="cuda") < case["masked"]] = -1
    return expert.contiguous()


def _combine_inputs(case, seed):
    """Result rows in the order of their experts, the place of each token's rows among them, and the weights."""
    g = _generator(seed)
    n, k, cols = case["tokens"], case["k"], case["cols"]
    rows = torch.randn((n * k, cols), generator=g, device="cuda").to(_TYPES[case["dtype"]])
    slot = torch.randperm(n * k, generator=g, device="cuda").to(torch.int32).view(n, k)
    slot[torch.rand(n, generator=g, device="cuda") < case["masked"]] = -1
    weight = torch.rand((n, k), generator=g, device="cuda") + 0.05
    weight /= weight.sum(dim=1, keepdim=True)
    base = torch.randn((n, cols), generator=g, device="cuda").to(_TYPES[case["out"]]) if case["base"] else None
    return rows, slot, weight, base


def _segments(case):
    """First row of each request, and the end of the last: ragged, from the case alone."""
    m, count = case["m"], min(case["requests"], case["m"])
    if count == m:
        return list(range(m + 1))
    rng = random.Random(7919 * m + count)
    return [0] + sorted(rng.sample(range(1, m), count - 1)) + [m]


def _adapters_inputs(case, seed):
    """Activations N(0, 1) with one channel in 64 twenty times as large; adapters whose share of the result is about a third of the projection's."""
    g = _generator(seed)
    m, n, k, r, e, s = case["m"], case["n"], case["k"], case["rank"], case["adapters"], case["sel"]
    x = torch.randn((m, k), generator=g, device="cuda")
    x[:, torch.randperm(k, generator=g, device="cuda")[:k // 64]] *= 20.0
    x = x.to(torch.bfloat16)
    w = (0.02 * torch.randn((n, k), generator=g, device="cuda")).to(torch.bfloat16)
    bias = 0.1 * torch.randn(n, generator=g, device="cuda") if case["bias"] else None
    a = (torch.randn((e, r, k), generator=g, device="cuda") / math.sqrt(k)).to(torch.bfloat16)
    b = (0.0066 * math.sqrt(k / (r * s)) * torch.randn((e, n, r), generator=g, device="cuda")).to(torch.bfloat16)
    if case["who"] == "router":
        which = torch.rand((m, e), generator=g, device="cuda").topk(s, dim=1).indices.to(torch.int32)
        weight = torch.rand((m, s), generator=g, device="cuda") + 0.05
        weight /= weight.sum(dim=1, keepdim=True)
    else:
        at = _segments(case)
        rng = random.Random(1000003 * seed + m)
        which = torch.empty((m, s), dtype=torch.int32)
        weight = torch.empty((m, s))
        for lo, hi in zip(at[:-1], at[1:]):
            which[lo:hi] = torch.tensor([-1 if rng.random() < 0.05 else i for i in rng.sample(range(e), s)], dtype=torch.int32)
            weight[lo:hi] = torch.tensor([rng.choice([0.5, 0.8, 1.0, 2.0]) for _ in range(s)])
        which, weight = which.cuda(), weight.cuda()
    return x, w, bias, a, b, which.contiguous(), weight.contiguous()


def prepare(case, seed):
    op = case["op"]
    s = {"op": op, "case": case}
    if own:
        from paper_2510_25590_amd import binding as rg
        s["ctx"] = rg.Context(256, 4, 64, 1024, 16, 16)
    if op == "route":
        s["logits"], s["bias"], s["mask"] = _route_inputs(case, seed)
        if own:
            s["expert"] = torch.zeros((case["tokens"], case["k"]), dtype=torch.int32, device="cuda")
            s["weight"] = torch.zeros((case["tokens"], case["k"]), device="cuda")
    elif op == "slots":
        s["expert"] = _slots_inputs(case, seed)
        if own:
            s["offsets"] = torch.zeros(case["experts"] + 1, dtype=torch.int32, device="cuda")
            s["row_token"] = torch.full((case["tokens"] * case["k"],), -1, dtype=torch.int32, device="cuda")
            s["slot"] = torch.zeros((case["tokens"], case["k"]), dtype=torch.int32, device="cuda")
    elif op == "combine":
        s["rows"], s["slot"], s["weight"], s["base"] = _combine_inputs(case, seed)
        if own:
            s["out"] = torch.zeros((case["tokens"], case["cols"]), dtype=_TYPES[case["out"]], device="cuda")
    else:
        s["x"], s["w"], s["bias"], s["a"], s["b"], s["which"], s["weight"] = _adapters_inputs(case, seed)
        if own:
            s["wp"] = rg.pack_weight(s["ctx"], s["w"])
            s["ap"] = rg.pack_adapters(s["ctx"], s["a"], s["b"])
            s["y"] = torch.zeros((case["m"], case["n"]), dtype=_TYPES[case["out"]], device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ plain forms


def _plain_route(s):
    c, logits = s["case"], s["logits"]
    n, e, k = c["tokens"], c["experts"], c["k"]
    l = logits.double()                                 # 64 bits: which of two experts with almost the same score is chosen
    if c["score"] == "softmax":
        score = torch.exp(l - l.amax(dim=1, keepdim=True))
        score = score / score.sum(dim=1, keepdim=True)
    else:
        score = 1.0 / (1.0 + torch.exp(-l))
    value = score + s["bias"].double() if s["bias"] is not None else score
    order = value if s["bias"] is not None else l       # without a bias the scores are in the order of the logits
    if c["groups"] > 1:
        best = value.view(n, c["groups"], -1).sort(dim=2, descending=True).values[:, :, :c["best"]].sum(dim=2)
        kept = best.sort(dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        keep = torch.zeros((n, c["groups"]), dtype=torch.bool, device=l.device)
        keep[torch.arange(n, device=l.device).unsqueeze(1), kept] = True
        order = torch.where(keep.repeat_interleave(e // c["groups"], dim=1), order, torch.full_like(order, -math.inf))
    expert = order.sort(dim=1, descending=True, stable=True).indices[:, :k]
    weight = torch.gather(score, 1, expert)
    if c["renorm"]:
        weight = weight / weight.sum(dim=1, keepdim=True)
    weight = (weight * c["scale"]).float()
    expert = expert.to(torch.int32)
    if s["mask"] is not None:
        out = (s["mask"] == 0).unsqueeze(1)
        expert, weight = expert.masked_fill(out, -1), weight.masked_fill(out, 0.0)
    return expert, weight


def _plain_slots(s):
    c = s["case"]
    flat = s["expert"].view(-1).long()
    key = torch.where(flat >= 0, flat, torch.full_like(flat, c["experts"]))
    order = key.sort(stable=True).indices
    counts = (key.unsqueeze(0) == torch.arange(c["experts"], device=key.device).unsqueeze(1)).sum(dim=1)
    offsets = torch.zeros(c["experts"] + 1, dtype=torch.int32, device=key.device)
    offsets[1:] = counts.cumsum(dim=0)
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=order.device)
    slot = torch.where(flat >= 0, place, torch.full_like(place, -1)).to(torch.int32).view(c["tokens"], c["k"])
    there = torch.arange(order.numel(), device=order.device) < offsets[-1]
    row_token = torch.where(there, torch.div(order, c["k"], rounding_mode="floor"), torch.full_like(order, -1)).to(torch.int32)
    return offsets, row_token, slot


def _plain_combine(s):
    c = s["case"]
    weight = torch.where(s["slot"] >= 0, s["weight"], torch.zeros_like(s["weight"]))
    at = s["slot"].clamp(min=0).long()
    out = s["base"].float() if s["base"] is not None else torch.zeros((c["tokens"], c["cols"]), device=at.device)
    for j in range(c["k"]):
        out = out + weight[:, j:j + 1] * s["rows"][at[:, j]].float()
    return out.to(_TYPES[c["out"]])


def _gelu(y):
    return 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))


def _plain_adapters(s):
    """All adapters side by side: their products with every row, times the row's weight of that adapter (0 for most)."""
    c, x = s["case"], s["x"].float()
    e, r = c["adapters"], c["rank"]
    share = ((s["which"].unsqueeze(2) == torch.arange(e, device=x.device)) * s["weight"].unsqueeze(2)).sum(dim=1)
    down = (x @ s["a"].float().view(e * r, -1).t()).view(-1, e, r) * share.unsqueeze(2)
    y = x @ s["w"].float().t() + down.view(-1, e * r) @ s["b"].float().transpose(1, 2).reshape(e * r, -1)
    if s["bias"] is not None:
        y = y + s["bias"]
    return (_gelu(y) if c["act"] == "gelu" else y).to(_TYPES[c["out"]])


_PLAIN = {"route": _plain_route, "slots": _plain_slots, "combine": _plain_combine, "adapters": _plain_adapters}


def run(s):
    if not own:
        return _PLAIN[s["op"]](s)
    from paper_2510_25590_amd import binding as rg
    c, ctx = s["case"], s["ctx"]
    code = {"bf16": rg.BF16, "f32": rg.FP32}
    if s["op"] == "route":
        rg.regione_expert_route(ctx, s["logits"], code[c["dtype"]], s["bias"], s["mask"], c["tokens"], c["experts"],
                                rg.SCORE_SOFTMAX if c["score"] == "softmax" else rg.SCORE_SIGMOID, c["groups"], c["top_groups"], c["best"], c["k"],
                                c["renorm"], c["scale"], s["expert"], s["weight"])
        return s["expert"], s["weight"]
    if s["op"] == "slots":
        rg.regione_expert_slots(ctx, s["expert"], c["tokens"], c["k"], c["experts"], s["offsets"], s["row_token"], s["slot"])
        return s["offsets"], s["row_token"], s["slot"]
    if s["op"] == "combine":
        rg.regione_expert_combine(ctx, s["rows"], code[c["dtype"]], c["tokens"] * c["k"], s["slot"], s["weight"], s["base"], c["tokens"], c["k"], c["cols"],
                                  code[c["out"]], s["out"])
        return s["out"]
    rg.regione_linear_adapters(ctx, s["x"], s["wp"], s["bias"], s["ap"], s["which"], s["weight"], c["adapters"], c["sel"], c["rank"], c["m"], c["n"], c["k"],
                               rg.ACT_GELU_TANH if c["act"] == "gelu" else rg.ACT_NONE, code[c["out"]], s["y"])
    return s["y"]


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits


def _exact_route(case, seed):
    logits, bias, mask = _route_inputs(case, seed)
    l = logits.double()
    n, e = l.shape
    score = torch.softmax(l, dim=1) if case["score"] == "softmax" else torch.sigmoid(l)
    value = score if bias is None else score + bias.double()
    rank_by = l.clone() if bias is None else value.clone()
    rows = torch.arange(n, device=l.device)
    if case["groups"] > 1:
        g, per = case["groups"], e // case["groups"]
        left = value.view(n, g, per).clone()
        total = torch.zeros((n, g), dtype=torch.float64, device=l.device)
        for _ in range(case["best"]):
            top = left.max(dim=2)
            total += top.values
            left.scatter_(2, top.indices.unsqueeze(2), -math.inf)
        open_group = torch.zeros((n, g), dtype=torch.bool, device=l.device)
        for _ in range(case["top_groups"]):
            index = torch.arange(g, device=l.device)
            at = torch.where(total == total.amax(dim=1, keepdim=True), index, torch.full_like(index, g)).amin(dim=1)
            open_group[rows, at] = True
            total[rows, at] = -math.inf
        rank_by = rank_by.view(n, g, per).masked_fill(~open_group.unsqueeze(2), -math.inf).view(n, e)
    expert, weight = [], []
    lowest = torch.arange(e, device=l.device)
    for _ in range(case["k"]):
        at = torch.where(rank_by == rank_by.amax(dim=1, keepdim=True), lowest, torch.full_like(lowest, e)).amin(dim=1)
        expert.append(at)
        weight.append(score[rows, at])
        rank_by[rows, at] = -math.inf
    expert, weight = torch.stack(expert, dim=1).to(torch.int32), torch.stack(weight, dim=1)
    if case["renorm"]:
        weight = weight / weight.sum(dim=1, keepdim=True)
    weight = weight * case["scale"]
    if mask is not None:
        expert[mask == 0] = -1
        weight[mask == 0] = 0.0
    return expert, weight


def _exact_slots(case, seed):
    expert = _slots_inputs(case, seed).cpu().view(-1).tolist()
    k = case["k"]
    of = [[] for _ in range(case["experts"])]
    for i, x in enumerate(expert):
        if x >= 0:
            of[x].append(i)
    offsets, row_token, slot = [0], [-1] * len(expert), [-1] * len(expert)
    for mine in of:
        for p, i in enumerate(mine, offsets[-1]):
            row_token[p], slot[i] = i // k, p
        offsets.append(offsets[-1] + len(mine))
    up = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    return up(offsets), up(row_token), up(slot).view(case["tokens"], k)


def _exact_combine(case, seed):
    rows, slot, weight, base = _combine_inputs(case, seed)
    out = torch.zeros((case["tokens"], case["cols"]), dtype=torch.float64, device="cuda") if base is None else base.double()
    for j in range(case["k"]):
        there = (slot[:, j] >= 0).nonzero().squeeze(1)
        out.index_add_(0, there, rows.index_select(0, slot[there, j].long()).double() * weight[there, j].double().unsqueeze(1))
    return out


def _exact_adapters(case, seed):
    x, w, bias, a, b, which, weight = _adapters_inputs(case, seed)
    x = x.double()
    y = x @ w.double().t().contiguous()
    if bias is not None:
        y += bias.double()
    for j in range(case["sel"]):
        for i in range(case["adapters"]):
            there = (which[:, j] == i).nonzero().squeeze(1)
            if there.numel():
                down = x[there] @ a[i].double().t().contiguous() * weight[there, j].double().unsqueeze(1)
                y[there] += down @ b[i].double().t().contiguous()
    return y * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)) if case["act"] == "gelu" else y


def exact(case, seed):
    return {"route": _exact_route, "slots": _exact_slots, "combine": _exact_combine, "adapters": _exact_adapters}[case["op"]](case, seed)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without


def work(case):
    size = {"bf16": 2.0, "f32": 4.0}
    if case["op"] == "route":
        n, e, k = case["tokens"], case["experts"], case["k"]
        routed = n * (1.0 - case["masked"])
        return {"bytes": routed * e * size[case["dtype"]] + (4.0 * e if case["bias"] else 0.0) + (n if case["masked"] else 0) + 8.0 * n * k, "flops": routed * e * 8.0}
    if case["op"] == "slots":
        return {"bytes": 12.0 * case["tokens"] * case["k"] + 4.0 * (case["experts"] + 1), "flops": 2.0 * case["tokens"] * case["k"]}
    if case["op"] == "combine":
        n, k, cols = case["tokens"], case["k"], case["cols"]
        used = n * k * (1.0 - case["masked"])
        return {"bytes": used * cols * size[case["dtype"]] + n * cols * size[case["out"]] * (2.0 if case["base"] else 1.0) + 8.0 * n * k, "flops": 2.0 * used * cols}
    m, n, k, r, s = case["m"], case["n"], case["k"], case["rank"], case["sel"]
    used = min(case["adapters"], s * (min(case["requests"], m) if case["who"] == "requests" else m))
    return {"bytes": 2.0 * m * k + 2.0 * n * k + 2.0 * used * r * (n + k) + 8.0 * m * s + (4.0 * n if case["bias"] else 0.0) + m * n * size[case["out"]],
            "flops": 2.0 * m * n * k + 2.0 * m * s * r * (n + k)}
