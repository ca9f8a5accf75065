"""Every tile of the 4-bit and the grouped products, forced, on sums that float32 holds exactly: sizes around the tile's own, K splits, results out of alignment, groups."""
import numpy as np
import pytest
import torch

from oracle import mx_reference as mx
from paper_2510_25590_amd import binding as rg

pytestmark = pytest.mark.gpu

TILES = [1, 2, 4, 8, 9, 72, 62, 52, 42, 32, 51, 41, 31, 22, 21, 11]


@pytest.fixture
def ctx():
    c = rg.Context(256, 4, 64, 1024, 64, 64)
    yield c
    c.close()


def up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def four_bit(ctx, rng, m, n, k):
    """Operands with scales of 1/2, 1 and 2 and exact sums: multiples of 1/16 below 36 * 4 k."""
    xc, wc = rng.integers(0, 16, (m, k)).astype(np.uint8), rng.integers(0, 16, (n, k)).astype(np.uint8)
    xs, ws = rng.integers(126, 129, (m, k // 32)).astype(np.uint8), rng.integers(126, 129, (n, k // 32)).astype(np.uint8)
    w = torch.empty(rg.regione_packed_weight_mxfp4_bytes(n, k), dtype=torch.uint8, device="cuda")
    rg.regione_pack_weight_mxfp4(ctx, up(mx.pack_codes(wc)), up(ws), n, k, w)
    return up(mx.pack_codes(xc)), up(mx.scale_steps(xs)), w, mx.values(xc, xs), mx.values(wc, ws)


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("m,n,k,splits", [(1, 8, 32, 1), (63, 65, 288, 1), (65, 264, 512, 1), (130, 200, 1024, 1), (257, 513, 800, 1), (300, 520, 1536, 2), (70, 136, 2560, 5), (513, 264, 3104, 3)])
def test_tiles(ctx, tile, m, n, k, splits):
    x, s, w, xv, wv = four_bit(ctx, np.random.default_rng(m + n + k), m, n, k)
    rg.regione_tune_mx(ctx, tile, splits)
    for offset in (0, 3):                       # of the result's first element: unaligned results go another way
        flat = torch.full((m * n + 16,), 0.3125, device="cuda")
        y = flat[offset:offset + m * n].view(m, n)
        for _ in range(2 if splits > 1 else 1): # the second run finds the arrival counters as the first left them
            rg.regione_linear_mxfp4(ctx, x, s, w, None, m, n, k, rg.ACT_NONE, rg.FP32, y)
            assert np.array_equal(y.cpu().double().numpy(), xv @ wv.T)
        assert (flat[:offset] == 0.3125).all() and (flat[offset + m * n:] == 0.3125).all()


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("fmt", ["mxfp4", "bf16"])
@pytest.mark.parametrize("sizes,first,m,n,k,use", [([0, 5, 64, 0, 129, 1], 0, 210, 136, 320, None), ([300, 11, 257], 7, 600, 328, 1024, [1, 0, 1]), ([3] * 100, 1, 310, 72, 128, [i % 6 for i in range(100)])])
def test_tiles_of_groups(ctx, tile, fmt, sizes, first, m, n, k, use):
    rng = np.random.default_rng(m + n)
    weights = 6 if use is None or max(use) > 1 else 2
    offsets = [first] + [int(v) for v in first + np.cumsum(sizes)]
    if fmt == "bf16":
        x = torch.from_numpy(rng.integers(-8, 9, (m, k)) / 4.0).float().to(torch.bfloat16)
        w = torch.from_numpy(rng.integers(-8, 9, (weights, n, k)) / 4.0).float().to(torch.bfloat16)
        wp = torch.stack([rg.pack_weight(ctx, w[i].cuda()) for i in range(weights)])
        xv, wv, xd = x.double().numpy(), w.double().numpy(), x.cuda()
    else:
        parts = [four_bit(ctx, rng, m, n, k) for _ in range(weights)]
        xd, s, xv = parts[0][0], parts[0][1], parts[0][3]
        wp, wv = torch.stack([p[2] for p in parts]), [p[4] for p in parts]
    o = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    u = None if use is None else torch.tensor(use, dtype=torch.int32, device="cuda")
    bias = rng.integers(-4, 5, (weights, n)).astype(np.float32)
    y = torch.full((m, n), 0.3125, device="cuda")
    rg.regione_tune_mx(ctx, tile)
    args = (wp, up(bias), o, u, len(sizes), weights, m, n, k, rg.ACT_NONE, rg.FP32, y)
    if fmt == "bf16":
        rg.regione_linear_grouped(ctx, xd, *args)
    else:
        rg.regione_linear_mxfp4_grouped(ctx, xd, s, *args)
    want = mx.grouped(xv, wv, bias, offsets, use, np.full((m, n), 0.3125))
    assert np.array_equal(y.cpu().double().numpy(), want)


@pytest.mark.parametrize("tile", [t for t in TILES if t > 9])
@pytest.mark.parametrize("act,out,offset", [(False, torch.bfloat16, 0), (True, torch.bfloat16, 0), (True, torch.float32, 0), (True, torch.bfloat16, 3), (True, torch.float32, 1)])
@pytest.mark.parametrize("n", [264, 261])
def test_k_splits_with_bias_and_activation(ctx, tile, act, out, offset, n):
    """Sums and bias are exact (multiples of 1/16); the activation is off by 2^-18 of its argument at most (tests/test_gpu_mxfp4.py), then the rounding to the result's type."""
    m, k = 150, 2080
    rng = np.random.default_rng(n)
    x, s, w, xv, wv = four_bit(ctx, rng, m, n, k)
    bias = rng.integers(-64, 65, n).astype(np.float32) / 16
    rg.regione_tune_mx(ctx, tile, 3)
    flat = torch.full((m * n + 16,), 0.3125, dtype=out, device="cuda")
    rg.regione_linear_mxfp4(ctx, x, s, w, up(bias), m, n, k, rg.ACT_GELU_TANH if act else rg.ACT_NONE, rg.FP32 if out == torch.float32 else rg.BF16, flat[offset:])
    z = xv @ wv.T + bias
    want = mx.gelu_tanh(z) if act else z
    bound = (2.0 ** -18 * np.abs(z) if act else 0.0) * (1 + torch.finfo(out).eps) + torch.finfo(out).eps / 2 * np.abs(want) + 2.0 ** -140
    got = flat[offset:offset + m * n].view(m, n).cpu().double().numpy()
    assert np.max(np.abs(got - want) / bound) <= 1.0
    assert (flat[:offset] == 0.3125).all() and (flat[offset + m * n:] == 0.3125).all()


def test_captured_k_split_replayed():
    """Replays with other rows each time, eager products of the same context between them: the sums and counters that K splits meet in are left ready by every call."""
    m, n, k = 130, 520, 4096
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = rg.Context(256, 4, 64, 1024, 64, 64, stream=stream)
        rng = np.random.default_rng(2)
        x, s, w, _, wv = four_bit(ctx, rng, m, n, k)
        y, z = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
        rg.regione_tune_mx(ctx, 21, 4)
        call = lambda to: rg.regione_linear_mxfp4(ctx, x, s, w, None, m, n, k, rg.ACT_NONE, rg.FP32, to)
        call(y)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call(y)
        for _ in range(4):
            codes, scale = rng.integers(0, 16, (m, k)).astype(np.uint8), rng.integers(126, 129, (m, k // 32)).astype(np.uint8)
            x.copy_(up(mx.pack_codes(codes)))
            s.copy_(up(mx.scale_steps(scale)))
            y.fill_(0.3125)
            graph.replay()
            call(z)
            stream.synchronize()
            want = mx.values(codes, scale) @ wv.T
            assert np.array_equal(y.cpu().double().numpy(), want) and np.array_equal(z.cpu().double().numpy(), want)
        ctx.close()


def test_two_contexts_at_once():
    """Contexts on streams of their own share nothing: products with K splits of both, launched alternately."""
    sides = []
    for i in range(2):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            ctx = rg.Context(256, 4, 64, 1024, 64, 64, stream=stream)
            m, n, k = 200 + 60 * i, 264, 5120
            x, s, w, xv, wv = four_bit(ctx, np.random.default_rng(i), m, n, k)
            rg.regione_tune_mx(ctx, 11, 8)
            ys = [torch.empty(m, n, device="cuda") for _ in range(10)]
            sides.append((ctx, stream, (x, s, w, None, m, n, k, rg.ACT_NONE, rg.FP32), ys, xv @ wv.T))
    torch.cuda.synchronize()
    for r in range(10):
        for ctx, stream, args, ys, _ in sides:
            rg.regione_linear_mxfp4(ctx, *args, ys[r])
    torch.cuda.synchronize()
    for ctx, _, _, ys, want in sides:
        assert all(np.array_equal(y.cpu().double().numpy(), want) for y in ys)
        ctx.close()
