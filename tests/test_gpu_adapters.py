"""Products with low-rank adapters beside them, through the C ABI, against oracle/expert_reference.py in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import expert_reference as ex
from paper_2510_25590_amd import binding as rg

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return rg.Context(256, 4, 64, 1024, 64, 64)


def up(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def of_rows(kind, rng, m, sel, count):
    """Adapters of the rows: of requests one after the other, of a router, none, or anything (numbers that no adapter has, one twice in a row)."""
    if kind == "requests":
        w = np.repeat(rng.integers(-1, count, (m, sel)), rng.integers(1, 40, m), axis=0)[:m]
    elif kind == "router":
        w = rng.integers(0, count, (m, sel))
    elif kind == "none":
        w = np.full((m, sel), -1)
    else:
        w = rng.choice([-2 ** 31, -1, 0, count - 1, count, 2 ** 31 - 1], (m, sel))
        w[:, -1] = w[:, 0]
    return w.astype(np.int32)


class Operands:
    def __init__(self, ctx, m, n, k, rank, count, sel, kind, seed, whole):
        """whole: small whole numbers (and weights of 1/2, 1, 2), whose sums float32 and the terms of the inner products hold exactly."""
        rng = np.random.default_rng(seed)
        self.m, self.n, self.k, self.rank, self.count, self.sel = m, n, k, rank, count, sel
        if whole:
            x, w, a, b = rng.integers(-2, 3, (m, k)), rng.integers(-2, 3, (n, k)), rng.integers(-1, 2, (count, rank, k)), rng.integers(-2, 3, (count, n, rank))
            self.weight = rng.choice([0.5, 1.0, 2.0], (m, sel)).astype(np.float32)
        else:
            x, w, a, b = rng.normal(size=(m, k)), 0.05 * rng.normal(size=(n, k)), rng.normal(size=(count, rank, k)) / np.sqrt(k), 0.5 * rng.normal(size=(count, n, rank))
            self.weight = rng.normal(size=(m, sel)).astype(np.float32)
        self.x, self.w, self.a, self.b = (torch.from_numpy(np.asarray(v, np.float32)).to(torch.bfloat16) for v in (x, w, a, b))
        self.which = of_rows(kind, rng, m, sel, count)
        self.xd, self.wp, self.ap = self.x.cuda(), rg.pack_weight(ctx, self.w.cuda()), rg.pack_adapters(ctx, self.a.cuda(), self.b.cuda())
        self.whichd, self.weightd = up(self.which), up(self.weight)

    def call(self, ctx, y, bias=None, act=False, weighted=True):
        rg.regione_linear_adapters(ctx, self.xd, self.wp, None if bias is None else up(bias), self.ap, self.whichd, self.weightd if weighted else None, self.count, self.sel, self.rank,
                                   self.m, self.n, self.k, rg.ACT_GELU_TANH if act else rg.ACT_NONE, rg.FP32 if y.dtype == torch.float32 else rg.BF16, y)
        return y

    def reference(self, bias=None, weighted=True):
        x, w, a, b = (v.double().numpy() for v in (self.x, self.w, self.a, self.b))
        weight = self.weight if weighted else None
        y, size = ex.adapters(x, w, bias, a, b, self.which, weight)
        return y, size, ex.adapters(x, np.zeros_like(w), None, a, b, self.which, weight)[1]


SHAPES = [  # m, n, k, rank, adapters, per row
    (1, 8, 64, 1, 1, 1), (1, 9216, 256, 16, 4, 1), (3, 40, 128, 7, 2, 2), (16, 64, 320, 16, 70, 1), (17, 65, 64, 17, 3, 3), (48, 520, 192, 8, 48, 1), (130, 264, 1024, 33, 5, 2),
    (300, 1032, 128, 64, 3, 1), (257, 130, 512, 100, 4, 2), (700, 96, 64, 256, 2, 1), (1100, 384, 256, 16, 8, 2), (4200, 72, 128, 20, 6, 3), (90, 3, 64, 5, 2, 1),
]


@pytest.mark.parametrize("kind", ["requests", "router", "none", "anything"])
@pytest.mark.parametrize("m,n,k,rank,count,sel", SHAPES)
def test_whole_numbers_exactly(ctx, m, n, k, rank, count, sel, kind):
    """Inner products below 2^12 in two or three terms of eight bits; sums below 2^23 / 2 in halves: exact whatever the order."""
    o = Operands(ctx, m, n, k, rank, count, sel, kind, m + n, True)
    bias = np.random.default_rng(1).integers(-9, 10, n).astype(np.float32)
    want = o.reference(bias)[0]
    assert np.max(np.abs(want)) < 2 ** 22
    assert np.array_equal(o.call(ctx, torch.full((m, n), 7.0, device="cuda"), bias).cpu().double().numpy(), want)
    low = o.call(ctx, torch.full((m, n), 7.0, dtype=torch.bfloat16, device="cuda"), bias)
    assert torch.equal(low.cpu(), torch.from_numpy(want).float().to(torch.bfloat16))


@pytest.mark.parametrize("act,out", [(False, torch.bfloat16), (True, torch.bfloat16), (False, torch.float32), (True, torch.float32)])
@pytest.mark.parametrize("m,n,k,rank,count,sel", SHAPES)
def test_values(ctx, act, out, m, n, k, rank, count, sel):
    """Float32 sums over the inputs (k) and over the adapters' terms, each at most the sizes' sum times 2^-24; the inner products' terms leave 2^-16 (two) or 2^-24 (three) of an adapter's
    share; the activation's slope and rounding as in the other products' tests; the output's rounding."""
    kind = ["requests", "router"][(m + n) % 2]
    o = Operands(ctx, m, n, k, rank, count, sel, kind, m * 3 + n, False)
    bias = np.random.default_rng(2).normal(size=n).astype(np.float32)
    z, size, share = o.reference(bias)
    terms = 3 if out == torch.float32 else 2
    err = (k + sel * terms * (rank + 16) + 8) * 2.0 ** -24 * size + 2.0 ** (-8 * terms) * share
    want = z
    if act:
        want, err = ex.gelu_tanh(z), 1.13 * err + 2.0 ** -18 * np.abs(z)
    err = err + torch.finfo(out).eps / 2 * (np.abs(want) + err) + 2.0 ** -140
    got = o.call(ctx, torch.full((m, n), 7.0, dtype=out, device="cuda"), bias, act).cpu().double().numpy()
    assert np.max(np.abs(got - want) / err) <= 1.0


TILES = (222, 224, 242, 244, 274, 284, 426, 436, 446, 44, 64, 74, 84, 266, 276)


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("tile", TILES)
def test_every_tile(tile, splits):
    """Whatever tile a product gets, with K splits and without, odd widths too."""
    ctx = rg.Context(256, 4, 64, 1024, 64, 64)
    rg.regione_tune_gemm(ctx, tile, splits)
    for n, kind in ((520, "requests"), (267, "router")):
        o = Operands(ctx, 300, n, 640, 24, 5, 2, kind, tile, True)
        assert np.array_equal(o.call(ctx, torch.empty(300, n, device="cuda")).cpu().double().numpy(), o.reference()[0])
    ctx.close()


@pytest.mark.parametrize("k", [64, 128, 192, 256])
@pytest.mark.parametrize("tile", TILES)
def test_products_shorter_than_their_pipeline(tile, k):
    """One to four steps of K, so that the copies ahead are the adapters' from the start, then or later; 0 to 15 steps of adapters."""
    ctx = rg.Context(256, 4, 64, 1024, 64, 64)
    rg.regione_tune_gemm(ctx, tile, 1)
    for rank, kind in ((16, "none"), (5, "requests"), (40, "router"), (64, "requests")):
        o = Operands(ctx, 270, 200, k, rank, 4, 2, kind, tile + k, True)
        for out in (torch.float32, torch.bfloat16):
            want = torch.from_numpy(o.reference()[0]).float().to(out)
            assert torch.equal(o.call(ctx, torch.empty(270, 200, dtype=out, device="cuda")).cpu(), want)
    ctx.close()


def test_without_weights_they_are_one(ctx):
    o = Operands(ctx, 70, 96, 128, 16, 3, 2, "router", 5, True)
    assert np.array_equal(o.call(ctx, torch.empty(70, 96, device="cuda"), weighted=False).cpu().double().numpy(), o.reference(weighted=False)[0])


@pytest.mark.parametrize("m,n", [(20, 64), (40, 2048), (300, 520), (2000, 1024)])
def test_rows_without_adapters_are_the_plain_product(ctx, m, n):
    """... bit for bit, where the plain product takes the same kernel; and adapters, rows and weights that are not finite reach no other row."""
    k = 256
    o = Operands(ctx, m, n, k, 16, 4, 1, "router", 6, False)
    o.which[::3] = -1
    o.whichd = up(o.which)
    y, plain = o.call(ctx, torch.empty(m, n, device="cuda")), torch.empty(m, n, device="cuda")
    rg.regione_linear(ctx, o.xd, o.wp, None, m, n, k, rg.ACT_NONE, rg.FP32, plain)
    assert torch.equal(y[::3], plain[::3])
    a, b = o.a.clone(), o.b.clone()
    a[1, 3, 5], b[1, 7, 2], b[2, 0, 0], b[2, n - 1, 15] = float("nan"), float("inf"), float("-inf"), float("nan")
    o.ap = rg.pack_adapters(ctx, a.cuda(), b.cuda())
    o.xd = o.xd.clone()
    o.xd[4] = float("inf")
    o.xd[5, 3] = float("nan")
    o.weightd[7] = float("nan")
    z = o.call(ctx, torch.empty(m, n, device="cuda"))
    touched = np.isin(o.which[:, 0], [1, 2])
    touched[[4, 5]] = True
    touched[7] = touched[7] or o.which[7, 0] >= 0
    assert torch.equal(z[~torch.from_numpy(touched).cuda()], y[~torch.from_numpy(touched).cuda()])
    # and only the columns that hold the values that are not finite
    rows = torch.from_numpy((o.which[:, 0] == 2) & (np.arange(m) != 4) & (np.arange(m) != 5) & (np.arange(m) != 7)).cuda()
    assert torch.equal(z[rows][:, 1:n - 1], y[rows][:, 1:n - 1]) and not torch.isfinite(z[rows][:, [0, n - 1]]).any()


def test_more_inner_products_than_are_kept_at_a_time(ctx):
    """32 adapters of rank 256 per row, float32: 1360 rows at a time."""
    o = Operands(ctx, 1500, 64, 64, 256, 40, 32, "router", 7, True)
    o.which[:, 8:] = -1                                                  # (the reference's time)
    o.which[:, 31] = 39
    o.whichd = up(o.which)
    assert np.array_equal(o.call(ctx, torch.empty(1500, 64, device="cuda")).cpu().double().numpy(), o.reference()[0])


@pytest.mark.parametrize("kind", ["requests", "router", "anything"])
@pytest.mark.parametrize("m,n,k,rank,count,sel", [(3000, 64, 192, 40, 5, 2), (600, 7, 128, 256, 3, 1), (8704, 33, 64, 16, 4, 1), (530, 64, 64, 9, 100, 5), (4097, 1, 320, 33, 7, 3)])
def test_narrow_results_of_many_rows(ctx, m, n, k, rank, count, sel, kind):
    """... which the kernel of 16 rows takes; whole numbers, and nothing behind the last row."""
    o = Operands(ctx, m, n, k, rank, count, sel, kind, m + n, True)
    for out in (torch.float32, torch.bfloat16):
        room = torch.full((m + 1, n), 7.0, dtype=out, device="cuda")
        o.call(ctx, room[:m])
        assert torch.equal(room[:m].cpu(), torch.from_numpy(o.reference()[0]).float().to(out)) and (room[m] == 7).all()


@pytest.mark.parametrize("count,sel", [(600, 1), (5000, 4), (20000, 16)])
def test_many_adapters_in_a_tile(ctx, count, sel):
    """Tiles that may name more adapters than the workspace has room for: passes over the rows, of few tiles, and the kernel of 16 rows."""
    m, n, k = 4200, 2304, 128
    o = Operands(ctx, m, n, k, 8, 8, sel, "router", 8, True)
    rng = np.random.default_rng(3)
    ids = np.sort(rng.choice(count, 8, replace=False))
    packed = torch.zeros(count, o.ap.shape[1], dtype=torch.bfloat16, device="cuda")
    packed[torch.from_numpy(ids).cuda()] = o.ap
    which = ids[o.which]
    which[::7] = rng.integers(0, count, which[::7].shape)                # adapters of zeros, but for the eight
    o.ap, o.whichd, o.count = packed, up(which.astype(np.int32)), count
    at = np.searchsorted(ids, which).clip(0, 7)
    o.which = np.where(ids[at] == which, at, -1).astype(np.int32)
    y = o.call(ctx, torch.full((m, n), 7.0, device="cuda"))
    assert np.array_equal(y.cpu().double().numpy(), o.reference()[0])


def test_adapters_past_32_bits(ctx):
    """3000 adapters of 1.5 MB: offsets past 2^31 elements."""
    n, k, rank, count = 9216, 3072, 64, 3000
    elems = rg.regione_packed_adapter_elems(n, k, rank)
    assert elems * count > 2 ** 31
    rng = np.random.default_rng(9)
    packed = torch.full((count, elems), float("nan"), dtype=torch.bfloat16, device="cuda")
    ids = [0, 2730, 2999]
    a, b = rng.integers(-1, 2, (3, rank, k)), rng.integers(-1, 2, (3, n, rank))
    packed[ids] = rg.pack_adapters(ctx, up(a, torch.bfloat16), up(b, torch.bfloat16))
    x = rng.integers(-1, 2, (3, k))
    which = torch.tensor([[i] for i in ids], dtype=torch.int32, device="cuda")
    y = torch.empty(3, n, device="cuda")
    rg.regione_linear_adapters(ctx, up(x, torch.bfloat16), torch.zeros(rg.regione_packed_weight_elems(n, k), dtype=torch.bfloat16, device="cuda"), None, packed, which, None, count, 1, rank, 3, n, k,
                               rg.ACT_NONE, rg.FP32, y)
    assert np.array_equal(y.cpu().numpy(), np.stack([b[i] @ (a[i] @ x[i]) for i in range(3)]))


def test_captured_and_replayed_with_other_adapters():
    """A captured call reads adapters and weights when it runs; eager calls of the same context's stream between the replays."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = rg.Context(256, 4, 64, 1024, 64, 64, stream=stream)
        for m, n, k in ((12, 128, 256), (600, 768, 512), (820, 1024, 4096)):
            o = Operands(ctx, m, n, k, 16, 6, 2, "requests", m, True)
            y = torch.zeros(m, n, device="cuda")
            o.call(ctx, y)
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                rg.regione_linear_adapters(ctx, o.xd, o.wp, None, o.ap, o.whichd, o.weightd, o.count, o.sel, o.rank, m, n, k, rg.ACT_NONE, rg.FP32, y)
            for seed in range(3):
                o.which = of_rows(["router", "none", "requests"][seed], np.random.default_rng(seed), m, 2, 6)
                o.whichd.copy_(up(o.which))
                y.fill_(7.0)
                graph.replay()
                got = y.cpu().double().numpy()
                assert np.array_equal(got, o.reference()[0])
                o.call(ctx, y.fill_(7.0))
                assert np.array_equal(y.cpu().double().numpy(), got)
            del graph
        ctx.close()


@pytest.mark.parametrize("m,n", [(5, 72), (300, 520), (300, 267)])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_results_at_any_address(ctx, m, n, out):
    """... and nothing beside them is written."""
    o = Operands(ctx, m, n, 192, 12, 3, 2, "router", m + n, True)
    for shift in (0, 1, 3):
        room = torch.full((m * n + 16,), 7.0, dtype=out, device="cuda")
        o.call(ctx, room[shift:shift + m * n].view(m, n))
        want = torch.from_numpy(o.reference()[0]).float().to(out)
        assert torch.equal(room[shift:shift + m * n].view(m, n).cpu(), want)
        assert (room[:shift] == 7).all() and (room[shift + m * n:] == 7).all()


@pytest.mark.parametrize("m", [7, 40, 700])
def test_the_most_adapters(ctx, m):
    """65536 of them, the first and the last named."""
    n, k, rank, count = 40, 64, 3, 65536
    o = Operands(ctx, m, n, k, rank, 3, 2, "router", 11, True)
    ids = np.array([0, 40000, 65535])
    packed = torch.zeros(count, o.ap.shape[1], dtype=torch.bfloat16, device="cuda")
    packed[torch.from_numpy(ids).cuda()] = o.ap
    o.ap, o.whichd, o.count = packed, up(ids[o.which].astype(np.int32)), count
    got = o.call(ctx, torch.full((m, n), 7.0, device="cuda"))
    assert np.array_equal(got.cpu().double().numpy(), o.reference()[0])


def test_values_that_are_not_finite_where_tiles_mix(ctx):
    """Rank 256, every row with one of five adapters; one of them holds an infinity and a NaN in B, one a NaN in A."""
    m, n, k, rank = 600, 2304, 128, 256
    o = Operands(ctx, m, n, k, rank, 5, 1, "router", 13, True)
    b, a = o.b.clone(), o.a.clone()
    b[3, 5, 200], b[3, 2300, 17], a[1, 255, 127] = float("inf"), float("nan"), float("nan")
    o.ap = rg.pack_adapters(ctx, a.cuda(), b.cuda())
    want = torch.from_numpy(o.reference()[0]).float()
    for out in (torch.float32, torch.bfloat16):
        got = o.call(ctx, torch.empty(m, n, dtype=out, device="cuda")).cpu()
        bad = torch.zeros(m, n, dtype=torch.bool)
        bad[torch.from_numpy(o.which[:, 0] == 1)] = True
        three = torch.from_numpy(np.flatnonzero(o.which[:, 0] == 3))
        bad[three, 5] = bad[three, 2300] = True
        assert torch.equal(torch.isnan(got), bad)
        assert torch.equal(got[~bad], want.to(out)[~bad])


def test_two_graphs_of_one_context():
    """Both use the context's workspace; replayed in turn, with eager calls between them."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = rg.Context(256, 4, 64, 1024, 64, 64, stream=stream)
        jobs = []
        for m, n, k, count in ((700, 640, 512, 4), (300, 1032, 1024, 40)):
            o = Operands(ctx, m, n, k, 24, count, 2, "router", m, True)
            y = torch.zeros(m, n, device="cuda")
            o.call(ctx, y)
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                rg.regione_linear_adapters(ctx, o.xd, o.wp, None, o.ap, o.whichd, o.weightd, o.count, o.sel, o.rank, m, n, k, rg.ACT_NONE, rg.FP32, y)
            jobs.append((o, y, graph, o.reference()[0]))
        for i in (0, 1, 1, 0, 1, 0):
            o, y, graph, want = jobs[i]
            y.fill_(7.0)
            graph.replay()
            assert np.array_equal(y.cpu().double().numpy(), want)
            other, z, _, expected = jobs[1 - i]
            assert np.array_equal(other.call(ctx, z.fill_(7.0)).cpu().double().numpy(), expected)
        del jobs, graph
        ctx.close()


def test_two_contexts_at_once():
    """Each on a stream of its own, with its own workspace."""
    jobs = []
    for i in range(2):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            c = rg.Context(256, 4, 64, 1024, 64, 64, stream=s)
            o = Operands(c, 900, 640, 512, 32, 4, 2, "requests", 20 + i, True)
            jobs.append((s, c, o, torch.zeros(900, 640, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(5):
        for s, c, o, y in jobs:
            with torch.cuda.stream(s):
                o.call(c, y.fill_(0.0))
    torch.cuda.synchronize()
    for s, c, o, y in jobs:
        assert np.array_equal(y.cpu().double().numpy(), o.reference()[0])
        c.close()


@pytest.mark.parametrize("n", [1, 60, 700])
def test_mixture_of_low_rank_experts(ctx, n):
    """A router's experts and weights, as they are, are the adapters of a projection."""
    width, out, experts, k, rank = 256, 320, 8, 2, 16
    o = Operands(ctx, n, out, width, rank, experts, k, "none", n, False)
    rng = np.random.default_rng(n)
    wr = up(rng.normal(size=(experts, width)), torch.bfloat16)
    logits = torch.empty(n, experts, device="cuda")
    mask = (rng.random(n) < 0.8).astype(np.uint8)
    rg.regione_linear(ctx, o.xd, rg.pack_weight(ctx, wr), None, n, experts, width, rg.ACT_NONE, rg.FP32, logits)
    rg.regione_expert_route(ctx, logits, rg.FP32, None, up(mask), n, experts, rg.SCORE_SOFTMAX, 1, 1, 1, k, True, 1.0, o.whichd, o.weightd)
    y = o.call(ctx, torch.empty(n, out, device="cuda")).cpu().double().numpy()
    o.which, o.weight = ex.route(logits.cpu().double().numpy(), None, mask, "softmax", 1, 1, 1, k, True, 1.0)
    assert np.array_equal(o.whichd.cpu().numpy(), o.which)
    want, size, share = o.reference()
    assert np.all(np.abs(y - want) <= (width + 2 * 3 * 32 + 9) * 2.0 ** -24 * size + 2.0 ** -24 * share + 2.0 ** -24 * np.abs(want) + 2.0 ** -140)


def test_pack_adapters_on_another_stream():
    """What the packing makes belongs to the context's stream; a caller on another one gets it in order."""
    s = torch.cuda.Stream()
    ctx = rg.Context(256, 4, 64, 1024, 64, 64, stream=s)
    a, b = torch.randn(2, 16, 64, device="cuda").to(torch.bfloat16), torch.randn(2, 40, 16, device="cuda").to(torch.bfloat16)
    packed = rg.pack_adapters(ctx, a, b)
    other = rg.Context(256, 4, 64, 1024, 64, 64)
    assert torch.equal(packed, rg.pack_adapters(other, a, b))
    first = packed[0, :16 * 64].view(2, 64, 8)                           # A in fragments of 16 ranks x 32 inputs
    want = a[0].view(16, 2, 4, 8).permute(1, 2, 0, 3).reshape(2, 64, 8)
    assert torch.equal(first, want)
    ctx.close()
    other.close()
