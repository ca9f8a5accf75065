"""Every tile of the 4-bit and the grouped products, forced, on sums that float32 holds exactly: sizes around the tile's own, K splits, results out of alignment, groups."""
import numpy as np
import pytest
import torch

from oracle import mx_reference as mx
from paper_2510_25590_amd import binding as rg

pytestmark = pytest.mark.gpu

TILES = [1, 2, 4, 8, 72, 62, 52, 42, 32, 51, 41, 31, 22, 21, 11]


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
