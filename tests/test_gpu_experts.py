"""Routing to experts, the sort by expert and the weighted sum, through the C ABI, against oracle/expert_reference.py in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import expert_reference as ex
from paper_2510_25590_amd import binding as rg

pytestmark = pytest.mark.gpu

SCORES = {"softmax": rg.SCORE_SOFTMAX, "sigmoid": rg.SCORE_SIGMOID}


@pytest.fixture(scope="module")
def ctx():
    return rg.Context(256, 4, 64, 1024, 64, 64)


def up(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def route(ctx, logits, bias, mask, score, groups, top_groups, best, k, renorm, scale):
    n, e = logits.shape
    expert = torch.full((n, k), -9, dtype=torch.int32, device="cuda")
    weight = torch.full((n, k), -9.0, device="cuda")
    rg.regione_expert_route(ctx, logits, rg.FP32 if logits.dtype == torch.float32 else rg.BF16, bias, mask, n, e, SCORES[score], groups, top_groups, best, k, renorm, scale, expert, weight)
    return expert.cpu().numpy(), weight.cpu().double().numpy()


def check_route(ctx, logits, bias, mask, score, groups, top_groups, best, k, renorm, scale):
    """Experts equal.  Weights are formed in 64 bits and rounded once (2^-24); a softmax without bias, groups and renormalising has its sum of exponentials in float32: the rounded
    difference in each exponent (|d| 2^-24 of the term), the exponential (two units: 2^-22), and at most 38 additions of positive terms."""
    got_e, got_w = route(ctx, logits, None if bias is None else up(bias), None if mask is None else up(mask), score, groups, top_groups, best, k, renorm, scale)
    l = logits.cpu().double().numpy()
    want_e, want_w = ex.route(l, bias, mask, score, groups, top_groups, best, k, renorm, scale)
    assert np.array_equal(got_e, want_e), np.argwhere(got_e != want_e)[:5]
    rel = np.full((l.shape[0], 1), 2.0 ** -24 * (1 + 2.0 ** -20))
    if score == "softmax" and bias is None and groups == 1 and not renorm:
        with np.errstate(invalid="ignore"):
            d = np.minimum(np.where(np.isnan(l), -np.inf, l), ex.FLOAT32_MAX)
            d = d - d.max(axis=1, keepdims=True)
            d = np.where(np.isfinite(d), d, -200.0)
        p = np.exp(d)
        rel = rel + 2.0 ** -24 * (((np.abs(d) * p).sum(axis=1) / p.sum(axis=1))[:, None] + 4 + 38)
    assert np.all(np.abs(got_w - want_w) <= rel * np.abs(want_w) + 2.0 ** -150), np.max(np.abs(got_w - want_w) / np.maximum(np.abs(want_w), 1e-300))


ROUTES = [  # experts, groups, top groups, best, k
    (1, 1, 1, 1, 1), (8, 1, 1, 1, 2), (60, 1, 1, 1, 4), (64, 1, 1, 1, 6), (65, 1, 1, 1, 8), (128, 1, 1, 1, 8), (160, 8, 3, 1, 6), (256, 8, 4, 2, 8), (256, 1, 1, 1, 32), (72, 9, 4, 2, 5),
    (384, 1, 1, 1, 10), (333, 3, 2, 2, 7), (1024, 64, 7, 2, 16), (1023, 33, 5, 1, 8), (1000, 5, 2, 2, 9), (1024, 1, 1, 1, 3), (16, 16, 3, 2, 3), (17, 17, 9, 1, 9),
]


@pytest.mark.parametrize("score,use_bias,renorm", [("softmax", False, True), ("softmax", False, False), ("softmax", True, False), ("softmax", True, True), ("sigmoid", True, True), ("sigmoid", False, False)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("experts,groups,top_groups,best,k", ROUTES)
def test_route(ctx, dtype, score, use_bias, renorm, experts, groups, top_groups, best, k):
    rng = np.random.default_rng(experts + groups)
    n = 37
    logits = up(rng.normal(size=(n, experts)) * 1.5, torch.float32).to(dtype)
    bias = (0.2 * rng.normal(size=experts)).astype(np.float32) if use_bias else None
    check_route(ctx, logits, bias, None, score, groups, top_groups, best, k, renorm, 2.5)


@pytest.mark.parametrize("tokens", [1, 2, 3, 5, 64, 255, 1025])
def test_route_tokens_and_masks(ctx, tokens):
    rng = np.random.default_rng(tokens)
    logits = up(rng.normal(size=(tokens, 96)), torch.float32)
    mask = rng.integers(0, 3, tokens).astype(np.uint8)                   # any nonzero byte routes
    check_route(ctx, logits, None, mask, "softmax", 1, 1, 1, 5, True, 1.0)
    check_route(ctx, logits, None, np.zeros(tokens, np.uint8), "sigmoid", 4, 2, 2, 5, True, 1.0)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,top_groups,best", [(1, 1, 1), (4, 2, 2), (4, 2, 1)])
@pytest.mark.parametrize("use_bias", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_route_special_values(ctx, score, groups, top_groups, best, use_bias, renorm):
    """Rows of ties, NaN, infinities, the largest and smallest values, and with fewer experts than are asked for; a bias that takes experts out."""
    e, k = 24, 6
    rng = np.random.default_rng(3)
    l = rng.normal(size=(20, e)).astype(np.float32)
    l[0] = 0.0
    l[1] = -np.inf
    l[2] = np.nan
    l[3], l[3, 7] = -np.inf, 1.0
    l[4, ::2] = np.nan
    l[5, 3], l[5, 11] = np.inf, np.inf
    l[6] = 3.0e38 * np.sign(l[6])
    l[7] *= 40.0
    l[8] = -200.0 - np.arange(e)
    l[9] = 1e-30 * np.arange(e)
    l[10, 6:] = -np.inf
    l[11] = np.round(l[11])
    l[12] = -0.0
    l[12, ::3] = 0.0
    l[13] = 88.0 + np.arange(e) % 5
    l[14] = -1.0e4
    l[15, :18] = -np.inf
    bias = None
    if use_bias:
        bias = (0.3 * rng.normal(size=e)).astype(np.float32)
        bias[5], bias[9], bias[20] = -np.inf, np.nan, 4.0
    check_route(ctx, up(l), bias, None, score, groups, top_groups, best, k, renorm, 1.0)


def test_route_near_ties_are_decided_in_64_bits(ctx):
    """Values that float32 cannot tell apart: the scores of neighbouring float32 logits, with a bias of one value."""
    base = np.float32(1.0)
    l = np.full((8, 64), base, np.float32)
    for t in range(8):
        l[t, 10 + t] = np.nextafter(base, np.float32(2.0))
        l[t, 40 - t] = np.nextafter(base, np.float32(0.0))
    bias = np.full(64, 3.0, np.float32)
    check_route(ctx, up(l), bias, None, "sigmoid", 1, 1, 1, 4, True, 1.0)
    check_route(ctx, up(l), bias, None, "softmax", 8, 3, 2, 4, False, 1.0)


# ------------------------------------------------------------------------------------------------ the sort


def sort(ctx, expert, experts):
    n, k = expert.shape
    offsets = torch.full((experts + 1,), -5, dtype=torch.int32, device="cuda")
    row_token = torch.full((max(1, n * k),), -5, dtype=torch.int32, device="cuda")
    slot = torch.full((max(1, n), k), -5, dtype=torch.int32, device="cuda")
    rg.regione_expert_slots(ctx, expert, n, k, experts, offsets, row_token, slot)
    return offsets, row_token[:n * k], slot[:n]


@pytest.mark.parametrize("tokens,k,experts", [(0, 1, 4), (1, 1, 1), (1, 3, 7), (36, 2, 16), (333, 8, 60), (1000, 5, 256), (1024, 8, 128), (1025, 8, 1024), (4097, 2, 3), (9001, 6, 64), (700, 32, 1000)])
@pytest.mark.parametrize("kind", ["random", "none", "one", "outside"])
def test_slots(ctx, tokens, k, experts, kind):
    rng = np.random.default_rng(tokens + k)
    e = rng.integers(-1, experts, (tokens, k)).astype(np.int32)
    if kind == "none":
        e[:] = -1
    elif kind == "one":
        e[:] = experts // 2
    elif kind == "outside":
        e[rng.random((tokens, k)) < 0.3] = experts
        e[rng.random((tokens, k)) < 0.2] = -2 ** 31
        e[rng.random((tokens, k)) < 0.2] = 2 ** 31 - 1
    got = sort(ctx, up(e), experts)
    want = ex.slots(e, experts, np.full(tokens * k, -5))
    for g, w in zip(got, want):
        assert np.array_equal(g.cpu().numpy(), w)


@pytest.mark.parametrize("tokens,k,experts", [(70001, 8, 128), (300000, 4, 300), (1 << 21, 8, 1024)])
def test_slots_of_many_pairs(ctx, tokens, k, experts):
    rng = np.random.default_rng(k)
    e = np.minimum(rng.geometric(8.0 / experts, (tokens, k)).astype(np.int32) - 2, experts - 1)
    offsets, row_token, slot = sort(ctx, up(e), experts)
    key = np.where(e >= 0, e, experts).reshape(-1)
    order = np.argsort(key, kind="stable")
    there = int((e >= 0).sum())
    assert np.array_equal(offsets.cpu().numpy(), np.concatenate([[0], np.cumsum(np.bincount(key, minlength=experts + 1)[:experts])]))
    assert np.array_equal(row_token.cpu().numpy(), np.concatenate([order[:there] // k, np.full(e.size - there, -5)]))
    place = np.empty(e.size, np.int64)
    place[order] = np.arange(e.size)
    assert np.array_equal(slot.cpu().numpy().reshape(-1), np.where(key < experts, place, -1))


# ------------------------------------------------------------------------------------------------ the weighted sum


@pytest.mark.parametrize("rows_t,out_t", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16), (torch.float32, torch.float32)])
@pytest.mark.parametrize("tokens,k,cols", [(1, 1, 1), (3, 2, 7), (8, 2, 3072), (5, 3, 64), (130, 4, 1000), (77, 8, 513), (20, 32, 520), (64, 5, 4096)])
@pytest.mark.parametrize("base,weighted", [(False, True), (True, True), (True, False)])
def test_combine(ctx, rows_t, out_t, tokens, k, cols, base, weighted):
    """float32 sums of k products and the base in order: (k + 1) roundings of at most the sum of the terms' sizes; the output's rounding."""
    rng = np.random.default_rng(tokens + cols)
    n_rows = tokens * k
    rows = up(rng.normal(size=(n_rows, cols)), torch.float32).to(rows_t)
    slot = rng.permutation(n_rows).reshape(tokens, k).astype(np.int32)
    slot[rng.random((tokens, k)) < 0.2] = -1
    slot[rng.random((tokens, k)) < 0.05] = n_rows                        # past the rows: nothing
    slot[rng.random((tokens, k)) < 0.05] = 0                             # the same row for several
    weight = rng.normal(size=(tokens, k)).astype(np.float32) if weighted else None
    b = up(rng.normal(size=(tokens, cols)), torch.float32).to(out_t) if base else None
    want, size = ex.combine(rows.cpu().double().numpy(), slot, weight, None if b is None else b.cpu().double().numpy())
    out = torch.full((tokens, cols), 7.0, dtype=out_t, device="cuda")
    code = lambda t: rg.FP32 if t == torch.float32 else rg.BF16
    args = (code(rows_t), n_rows, up(slot), None if weight is None else up(weight))
    rg.regione_expert_combine(ctx, rows, *args, b, tokens, k, cols, code(out_t), out)
    err = (k + 1) * 2.0 ** -24 * size
    err += torch.finfo(out_t).eps / 2 * (np.abs(want) + err) + 2.0 ** -140
    assert np.all(np.abs(out.cpu().double().numpy() - want) <= err)
    if base:                                                             # into the base itself
        rg.regione_expert_combine(ctx, rows, *args, b, tokens, k, cols, code(out_t), b)
        assert torch.equal(b, out)


def test_combine_leaves_unused_rows_alone_and_is_unaligned(ctx):
    """Rows that no slot names may hold anything; tensors that start at odd elements take the narrow path with the same results."""
    tokens, k, cols = 33, 3, 72
    rng = np.random.default_rng(5)
    rows = up(rng.normal(size=(200, cols)), torch.bfloat16)
    slot = rng.integers(50, 150, (tokens, k)).astype(np.int32)
    slot[::4, 1] = -1
    rows[:50], rows[150:] = float("nan"), float("inf")
    weight = rng.random((tokens, k)).astype(np.float32)
    out = torch.empty(tokens, cols, dtype=torch.bfloat16, device="cuda")
    rg.regione_expert_combine(ctx, rows, rg.BF16, 200, up(slot), up(weight), None, tokens, k, cols, rg.BF16, out)
    assert torch.isfinite(out).all()
    store = torch.empty(200 * cols + 3, dtype=torch.bfloat16, device="cuda")
    odd = store[3:].view(200, cols)
    odd.copy_(rows)
    out2 = torch.empty(tokens, cols, dtype=torch.bfloat16, device="cuda")
    rg.regione_expert_combine(ctx, odd, rg.BF16, 200, up(slot), up(weight), None, tokens, k, cols, rg.BF16, out2)
    assert torch.equal(out, out2)


def test_combine_past_32_bits(ctx):
    """Rows whose elements lie past 2^31."""
    cols, n_rows = 4096, 600000
    rows = torch.zeros(n_rows, cols, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([[n_rows - 1, 0], [n_rows - 2, 524288], [524287, 524289], [3, 550001]], dtype=torch.int32, device="cuda")
    rows[at.flatten().long()] = torch.arange(1.0, 9.0, device="cuda").to(torch.bfloat16)[:, None]
    out = torch.empty(4, cols, device="cuda")
    rg.regione_expert_combine(ctx, rows, rg.BF16, n_rows, at, None, None, 4, 2, cols, rg.FP32, out)
    assert torch.equal(out, torch.tensor([3.0, 7.0, 11.0, 15.0], device="cuda")[:, None].expand(4, cols))


# ------------------------------------------------------------------------------------------------ together


def expert_layer(ctx, x, router, w1, w2, hidden, experts, k, residual):
    """A routed MLP as a program runs it; all sizes known to the host but the experts' rows."""
    n, width = x.shape
    new = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device="cuda")
    logits, expert, weight = new(n, experts), new(n, k, dtype=torch.int32), new(n, k)
    offsets, row_token, slot = new(experts + 1, dtype=torch.int32), torch.zeros(n * k, dtype=torch.int32, device="cuda"), new(n, k, dtype=torch.int32)
    rows, up_rows, down_rows, out = torch.zeros(n * k, width, dtype=torch.bfloat16, device="cuda"), new(n * k, hidden, dtype=torch.bfloat16), new(n * k, width), new(n, width)

    def run():
        rg.regione_linear(ctx, x, router, None, n, experts, width, rg.ACT_NONE, rg.FP32, logits)
        rg.regione_expert_route(ctx, logits, rg.FP32, None, None, n, experts, rg.SCORE_SOFTMAX, 1, 1, 1, k, True, 1.0, expert, weight)
        rg.regione_expert_slots(ctx, expert, n, k, experts, offsets, row_token, slot)
        rg.regione_gather(ctx, x, width, rg.BF16, row_token, offsets[experts:], n * k, rows)
        rg.regione_linear_grouped(ctx, rows, w1, None, offsets, None, experts, experts, n * k, hidden, width, rg.ACT_NONE, rg.BF16, up_rows)
        rg.regione_linear_grouped(ctx, up_rows, w2, None, offsets, None, experts, experts, n * k, width, hidden, rg.ACT_NONE, rg.FP32, down_rows)
        rg.regione_expert_combine(ctx, down_rows, rg.FP32, n * k, slot, weight, residual, n, k, width, rg.FP32, out)
    return run, out, expert, weight, logits


@pytest.mark.parametrize("n,width,hidden,experts,k", [(1, 128, 192, 8, 2), (50, 256, 320, 16, 4), (700, 192, 256, 12, 3)])
def test_routed_layer(n, width, hidden, experts, k):
    """Products of small whole numbers are exact, so that only the weights and their sum round; captured and replayed with other inputs, eager work between the replays."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = rg.Context(256, 4, 64, 1024, 64, 64, stream=stream)
        rng = np.random.default_rng(n)
        few = lambda *s: (rng.integers(-1, 2, s) * (rng.random(s) < 0.08)).astype(np.float32)
        w1, w2, wr = few(experts, hidden, width), few(experts, width, hidden), (rng.integers(-8, 9, (experts, width)) / 16.0).astype(np.float32)
        pack = lambda w: torch.stack([rg.pack_weight(ctx, up(w[i], torch.bfloat16)) for i in range(experts)])
        x, residual = torch.empty(n, width, dtype=torch.bfloat16, device="cuda"), torch.empty(n, width, device="cuda")
        run, out, expert, weight, logits = expert_layer(ctx, x, rg.pack_weight(ctx, up(wr, torch.bfloat16)), pack(w1), pack(w2), hidden, experts, k, residual)

        def fill(seed):
            g = np.random.default_rng(seed)
            xs, rs = g.integers(-2, 3, (n, width)).astype(np.float32), g.normal(size=(n, width)).astype(np.float32)
            x.copy_(up(xs, torch.bfloat16))
            residual.copy_(up(rs))
            return xs.astype(np.float64), rs.astype(np.float64)

        def check(xs, rs):
            want_e, want_w = ex.route(xs @ wr.T.astype(np.float64), None, None, "softmax", 1, 1, 1, k, True, 1.0)
            assert np.array_equal(expert.cpu().numpy(), want_e)
            want, size = rs.copy(), np.abs(rs)
            for t in range(n):
                for j in range(k):
                    mid = w1[want_e[t, j]].astype(np.float64) @ xs[t]
                    assert np.max(np.abs(mid)) <= 256                    # exact in bf16
                    term = want_w[t, j] * (w2[want_e[t, j]].astype(np.float64) @ mid)
                    want[t] += term
                    size[t] += np.abs(term)
            assert np.all(np.abs(out.cpu().double().numpy() - want) <= (k + 3) * 2.0 ** -24 * size + 2.0 ** -140)

        xs, rs = fill(100)
        run()
        stream.synchronize()
        check(xs, rs)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run()
        for seed in (101, 102, 103):
            xs, rs = fill(seed)
            graph.replay()
            stream.synchronize()
            check(xs, rs)
            replayed = out.clone()
            out.fill_(0.0)
            run()
            stream.synchronize()
            assert torch.equal(out, replayed)
        del graph
        ctx.close()


def test_float32_contexts_route_sort_and_combine():
    ctx = rg.Context(256, 4, 64, 1024, 64, 64, compute_dtype=rg.FP32)
    rng = np.random.default_rng(8)
    check_route(ctx, up(rng.normal(size=(40, 20)), torch.float32), None, None, "softmax", 1, 1, 1, 3, True, 1.0)
    e = rng.integers(0, 20, (5000, 3)).astype(np.int32)
    for g, w in zip(sort(ctx, up(e), 20), ex.slots(e, 20, np.full(15000, -5))):
        assert np.array_equal(g.cpu().numpy(), w)
    ctx.close()
