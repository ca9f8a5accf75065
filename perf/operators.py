"""What the 4-bit and the grouped products are timed on, and their plain forms.

Operators: quantisation of rows to microscaled 4-bit floating point (MXFP4: E2M1 values, one power of two per 32
values of a row) and back; the product of such rows with such weights; the same product over ragged groups of rows
that have weights of their own; and that grouped product in bf16.  Sizes are those of the repository's blocks (widths
256 and 3072, 820 or 1382 edited rows, 8704 rows of a full forward) and of generic expert layers.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 32                                              # values that share a scale
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)         # by code; bit 3 is the sign


# ------------------------------------------------------------------------------------------------ the cases


def listed():
    return [
        # A handful of float32 rows of the residual stream (eight edited tokens): launch latency.
        {"name": "quantize_8_rows_f32", "op": "quantize", "rows": 8, "cols": 3072, "dtype": "f32"},
        # The MLP rows of a full forward, 8704 tokens: HBM.
        {"name": "quantize_8704_mlp_rows", "op": "quantize", "rows": 8704, "cols": 12288, "dtype": "bf16"},
        # One row through a QKV projection (a single edited token): the weights from HBM.
        {"name": "linear_1_row_qkv", "op": "linear", "m": 1, "n": 9216, "k": 3072, "act": "none", "out": "bf16", "bias": True},
        # The 256-wide configuration, 36 edited rows, float32 result: launch latency.
        {"name": "linear_36_rows_w256", "op": "linear", "m": 36, "n": 768, "k": 256, "act": "none", "out": "f32", "bias": True},
        # MLP up of the benchmark block, 20 % of a 64x64 image edited.
        {"name": "linear_820_rows_mlp_up", "op": "linear", "m": 820, "n": 12288, "k": 3072, "act": "gelu", "out": "bf16", "bias": True},
        # The second product of a single-stream block ([attention | MLP] rows) of a 96x96 image, 15 % edited; float32 result.
        {"name": "linear_1382_rows_joint", "op": "linear", "m": 1382, "n": 3072, "k": 15360, "act": "none", "out": "f32", "bias": True},
        # QKV of a full forward: every row of the sequence.
        {"name": "linear_8704_rows_qkv", "op": "linear", "m": 8704, "n": 9216, "k": 3072, "act": "none", "out": "bf16", "bias": True},
        # Text and image rows of a double-stream block, weights of their own, in 4 bits.
        {"name": "grouped_text_image_4bit", "op": "grouped", "format": "mxfp4", "m": 1332, "groups": 2, "weights": 2, "n": 9216, "k": 3072,
         "act": "none", "out": "bf16", "spread": "ragged"},
        # An expert layer on few rows: most experts have one, two or none.
        {"name": "grouped_64_experts_96_rows_4bit", "op": "grouped", "format": "mxfp4", "m": 96, "groups": 64, "weights": 64, "n": 2048, "k": 1024,
         "act": "gelu", "out": "bf16", "spread": "ragged"},
        # An expert layer on many rows.
        {"name": "grouped_16_experts_16384_rows_4bit", "op": "grouped", "format": "mxfp4", "m": 16384, "groups": 16, "weights": 16, "n": 4096, "k": 2048,
         "act": "gelu", "out": "bf16", "spread": "ragged"},
        # Two guidance branches of a double-stream block in bf16: text and image rows alternate, two weights for four groups.
        {"name": "grouped_two_branches_bf16", "op": "grouped", "format": "bf16", "m": 2664, "groups": 4, "weights": 2, "n": 3072, "k": 3072,
         "act": "none", "out": "bf16", "spread": "ragged"},
        # An expert layer in bf16, float32 result.
        {"name": "grouped_16_experts_2000_rows_bf16", "op": "grouped", "format": "bf16", "m": 2000, "groups": 16, "weights": 16, "n": 2048, "k": 1024,
         "act": "gelu", "out": "f32", "spread": "ragged"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "linear", "grouped", "grouped", "grouped"])
    if op == "quantize":
        rows, cols = _log_int(rng, 1, 8704), BLOCK * _log_int(rng, 8, 384)
        return {"op": op, "rows": rows, "cols": cols, "dtype": rng.choice(["bf16", "f32"])}
    act, out = rng.choice(["none", "gelu"]), rng.choice(["bf16", "bf16", "f32"])
    if op == "linear":
        m = _log_int(rng, 1, 8704)
        n = _log_int(rng, 64, 9216) if rng.random() < 0.3 else 8 * _log_int(rng, 32, 1152)
        k = BLOCK * _log_int(rng, 8, 480 if m < 3000 else 96)
        return {"op": op, "m": m, "n": n, "k": k, "act": act, "out": out, "bias": rng.random() < 0.8}
    groups = rng.choice([1, 2, 4, 8, 16, 32, 64])
    fmt = rng.choice(["mxfp4", "mxfp4", "bf16"])
    m = _log_int(rng, 1, 16384)
    k = BLOCK * _log_int(rng, 8, 64) if fmt == "mxfp4" else 64 * _log_int(rng, 4, 32)
    return {"op": op, "format": fmt, "m": m, "groups": groups, "weights": groups if rng.random() < 0.7 else max(1, groups // 2),
            "n": 8 * _log_int(rng, 16, 384), "k": k, "act": act, "out": out, "spread": rng.choice(["ragged", "even", "one"])}


def _offsets(case):
    """First row of each group, and the end of the last: from the case alone."""
    g, m = case["groups"], case["m"]
    if case["spread"] == "even":
        return [m * i // g for i in range(g + 1)]
    if case["spread"] == "one":                         # everything in one group, the others are empty
        return [0 if i <= g // 2 else m for i in range(g + 1)]
    rng = random.Random(1000003 * m + g)
    share = [rng.expovariate(1.0) ** 1.5 for _ in range(g)]
    total, at, offsets = sum(share), 0.0, [0]
    for s in share:
        at += s
        offsets.append(min(m, int(m * at / total + 0.5)))
    offsets[-1] = m
    return offsets


# ------------------------------------------------------------------------------------------------ inputs


def _rows(g, rows, cols, dtype):
    """Activations: N(0, 1), one channel in 64 twenty times as large, one row in 16 a thousand times smaller."""
    x = torch.randn((rows, cols), generator=g, device="cuda")
    x[:, torch.randperm(cols, generator=g, device="cuda")[:cols // 64]] *= 20.0
    x[torch.randperm(rows, generator=g, device="cuda")[:rows // 16]] *= 1e-3
    return x.to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op = case["op"]
    if op == "quantize":
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        s = {"op": op, "x": _rows(g, case["rows"], case["cols"], dt)}
        if own:
            from paper_2510_25590_amd import binding as rg
            s["ctx"] = rg.Context(256, 4, 64, 1024, 16, 16)
            s["q"] = torch.zeros((case["rows"], case["cols"] // 2), dtype=torch.uint8, device="cuda")
            s["scale"] = torch.zeros(rg.regione_mxfp4_scale_bytes(case["rows"], case["cols"], rg.MX_SCALE_STEPS), dtype=torch.uint8, device="cuda")
            s["y"] = torch.zeros((case["rows"], case["cols"]), dtype=torch.bfloat16, device="cuda")
        return s
    m, n, k = case["m"], case["n"], case["k"]
    weights = case["weights"] if op == "grouped" else 1
    fmt = case["format"] if op == "grouped" else "mxfp4"
    x = _rows(g, m, k, torch.bfloat16)
    w = (0.02 * torch.randn((weights, n, k), generator=g, device="cuda")).to(torch.bfloat16)
    bias = 0.1 * torch.randn((weights, n), generator=g, device="cuda") if case.get("bias", True) else None
    out = torch.float32 if case["out"] == "f32" else torch.bfloat16
    s = {"op": op, "format": fmt, "act": case["act"], "out": out, "bias": bias, "n": n, "k": k, "m": m, "weights": weights}
    if op == "grouped":
        s["offsets_host"] = _offsets(case)
        s["offsets"] = torch.tensor(s["offsets_host"], dtype=torch.int32, device="cuda")
        s["use"] = [i % weights for i in range(case["groups"])]
        s["use_dev"] = torch.tensor(s["use"], dtype=torch.int32, device="cuda")
    if fmt == "mxfp4":
        s["xq"], s["xe"] = _codes(x)
        s["wq"], s["we"] = _codes(w.view(weights * n, k))
    else:
        s["x"], s["w"] = x, w
    if own:
        from paper_2510_25590_amd import binding as rg
        s["ctx"] = rg.Context(256, 4, 64, 1024, max(16, m), 16)
        if fmt == "mxfp4":
            s["q"], s["scale"] = rg.quantize_rows_mxfp4(s["ctx"], x)
            s["wp"] = torch.stack([rg.pack_weight_mxfp4(s["ctx"], w[i]) for i in range(weights)])
        else:
            s["wp"] = torch.stack([rg.pack_weight(s["ctx"], w[i]) for i in range(weights)])
        s["y"] = torch.zeros((m, n), dtype=out, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ plain forms


def _exponents(amax):
    """floor(log2 amax) - 2, not below -127 (float32 in, int32 out)."""
    return (torch.frexp(amax)[1] - 3).clamp(min=-127).where(amax > 0, torch.full((), -127, dtype=torch.int32, device=amax.device))


def _power(e):
    """2^e in float32 for whole e from -127 on, exact (exp2 is not)."""
    return torch.where(e < -126, torch.full_like(e, 1 << 22), (e + 127) << 23).view(torch.float32)


def _scaled(x):
    """Blocks of x divided by their scale, and the exponents of the scales."""
    b = x.float().view(x.shape[0], -1, BLOCK)
    e = _exponents(b.abs().amax(dim=2))
    # in two factors, since 2^-e by itself may not be a normal float32
    half = torch.div(-e, 2, rounding_mode="floor")
    return b * _power(half).unsqueeze(2) * _power(-e - half).unsqueeze(2), e


def _rounded(a):
    """Magnitudes to the nearest E2M1 value, ties to the even code."""
    step = 0.5 + 0.5 * (a >= 2.0).float() + (a >= 4.0).float()
    return torch.clamp(torch.round(a / step) * step, max=6.0)


def _codes(x):
    """Codes [rows, cols / 2], the value of the lower column in the lower four bits, and scale bytes [rows, cols / 32]."""
    v, e = _scaled(x)
    a = _rounded(v.abs())
    code = (a * 2.0 - (a - 2.0).clamp(min=0.0) - 0.5 * (a - 4.0).clamp(min=0.0)).to(torch.uint8) | ((v < 0).to(torch.uint8) << 3)
    code = code.view(x.shape[0], -1, 2)
    return code[:, :, 0] | (code[:, :, 1] << 4), (e + 127).to(torch.uint8)


def _values(q, e):
    """Float32 values of codes and scale bytes."""
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=torch.float32, device=q.device)
    pair = torch.stack((q & 15, q >> 4), dim=2).view(q.shape[0], -1, BLOCK)
    return (table[pair.int()] * _power(e.int() - 127).unsqueeze(2)).view(q.shape[0], -1)


def _gelu(y):
    return 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))


def _finish(y, bias, act, out):
    if bias is not None:
        y = y + bias
    return (_gelu(y) if act == "gelu" else y).to(out)


def _plain(s):
    if s["op"] == "quantize":
        v, e = _scaled(s["x"])
        return (torch.sign(v) * _rounded(v.abs()) * _power(e).unsqueeze(2)).view(s["x"].shape).to(torch.bfloat16)
    if s["op"] == "linear":
        y = _values(s["xq"], s["xe"]) @ _values(s["wq"], s["we"]).t()
        return _finish(y, None if s["bias"] is None else s["bias"][0], s["act"], s["out"])
    x = _values(s["xq"], s["xe"]) if s["format"] == "mxfp4" else s["x"].float()
    y = torch.zeros((s["m"], s["n"]), dtype=s["out"], device=x.device)
    for i, u in enumerate(s["use"]):
        lo, hi = s["offsets_host"][i], s["offsets_host"][i + 1]
        if lo < hi:
            w = _values(s["wq"][u * s["n"]:(u + 1) * s["n"]], s["we"][u * s["n"]:(u + 1) * s["n"]]) if s["format"] == "mxfp4" else s["w"][u].float()
            y[lo:hi] = _finish(x[lo:hi] @ w.t(), None if s["bias"] is None else s["bias"][u], s["act"], s["out"])
    return y


def run(s):
    if not own:
        return _plain(s)
    from paper_2510_25590_amd import binding as rg
    if s["op"] == "quantize":
        rows, cols = s["x"].shape
        dt = rg.FP32 if s["x"].dtype == torch.float32 else rg.BF16
        rg.regione_quantize_rows_mxfp4(s["ctx"], s["x"], dt, rows, cols, rg.MX_SCALE_STEPS, s["q"], s["scale"])
        rg.regione_dequantize_rows_mxfp4(s["ctx"], s["q"], s["scale"], rg.MX_SCALE_STEPS, rows, cols, rg.BF16, s["y"])
        return s["y"]
    act = rg.ACT_GELU_TANH if s["act"] == "gelu" else rg.ACT_NONE
    out = rg.FP32 if s["out"] == torch.float32 else rg.BF16
    if s["op"] == "linear":
        rg.regione_linear_mxfp4(s["ctx"], s["q"], s["scale"], s["wp"], s["bias"], s["m"], s["n"], s["k"], act, out, s["y"])
    elif s["format"] == "mxfp4":
        rg.regione_linear_mxfp4_grouped(s["ctx"], s["q"], s["scale"], s["wp"], s["bias"], s["offsets"], s["use_dev"], len(s["use"]), s["weights"],
                                        s["m"], s["n"], s["k"], act, out, s["y"])
    else:
        rg.regione_linear_grouped(s["ctx"], s["x"], s["wp"], s["bias"], s["offsets"], s["use_dev"], len(s["use"]), s["weights"],
                                  s["m"], s["n"], s["k"], act, out, s["y"])
    return s["y"]


# ------------------------------------------------------------------------------------------------ the definition, in 64 bits


def _exact_rows(x):
    """Values of x after quantisation: the nearest of all representable values, found by search."""
    d = x.double().view(-1, BLOCK)
    amax = d.abs().amax(dim=1, keepdim=True)
    _, e = torch.frexp(amax)                            # amax = f 2^e with f in [1/2, 1)
    e = torch.where(amax > 0, (e - 3).clamp(-127, 127), torch.full_like(e, -127))
    scale = ((e.long() + 1023) << 52).view(torch.float64)       # 2^e
    t = (d / scale).abs()
    got = torch.zeros_like(t)
    for lower, upper, even in zip(E2M1[:-1], E2M1[1:], range(7)):
        middle = (lower + upper) / 2
        up = t > middle if even % 2 == 0 else t >= middle
        got = torch.where(up, torch.full_like(t, upper), got)
    return (torch.copysign(got, d) * scale).view(x.shape)


def exact(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if case["op"] == "quantize":
        return _exact_rows(_rows(g, case["rows"], case["cols"], torch.float32 if case["dtype"] == "f32" else torch.bfloat16))
    m, n, k = case["m"], case["n"], case["k"]
    grouped = case["op"] == "grouped"
    weights = case["weights"] if grouped else 1
    x = _rows(g, m, k, torch.bfloat16)
    w = (0.02 * torch.randn((weights, n, k), generator=g, device="cuda")).to(torch.bfloat16)
    bias = 0.1 * torch.randn((weights, n), generator=g, device="cuda") if case.get("bias", True) else torch.zeros((weights, n), device="cuda")
    four = not grouped or case["format"] == "mxfp4"
    x = _exact_rows(x) if four else x.double()
    offsets = _offsets(case) if grouped else [0, m]
    y = torch.zeros((m, n), dtype=torch.float64, device="cuda")
    for i in range(len(offsets) - 1):
        rows, u = slice(offsets[i], offsets[i + 1]), i % weights
        if offsets[i] == offsets[i + 1]:
            continue
        z = torch.addmm(bias[u].double(), x[rows], (_exact_rows(w[u]) if four else w[u].double()).t().contiguous())
        if case["act"] == "gelu":
            z = z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))
        y[rows] = z
    return y


# ------------------------------------------------------------------------------------------------ what a pass cannot do without


def work(case):
    if case["op"] == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * ((4.0 if case["dtype"] == "f32" else 2.0) + 2.0), "flops": 2.0 * n}
    m, n, k = case["m"], case["n"], case["k"]
    el = 2.0 if case["op"] == "grouped" and case["format"] == "bf16" else 0.5 + 1.0 / BLOCK
    used = 1
    if case["op"] == "grouped":
        o = _offsets(case)
        used = len({i % case["weights"] for i in range(case["groups"]) if o[i] < o[i + 1]})
    return {"bytes": m * k * el + used * n * (k * el + 4.0) + m * n * (4.0 if case["out"] == "f32" else 2.0), "flops": 2.0 * m * n * k}
