"""Offsets that do not ascend: groups that share no row are right in any order; with shared rows, which the contract excludes, nothing else is written and every launch ends."""
import numpy as np
import pytest
import torch

from oracle import mx_reference as mx
from paper_2510_25590_amd import binding as rg

pytestmark = pytest.mark.gpu

UNTOUCHED = 0.3125


@pytest.fixture(scope="module")
def ctx():
    return rg.Context(256, 4, 64, 1024, 64, 64)


def up(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def operands(ctx, fmt, m, n, k, weights):
    """Sums that float32 holds exactly: multiples of 1/16 below 4 k, or of 1/4 below 36 k."""
    rng = np.random.default_rng(m + n)
    if fmt == "bf16":
        x, w = (torch.from_numpy(rng.integers(-8, 9, s) / 4.0).float().to(torch.bfloat16) for s in ((m, k), (weights, n, k)))
        packed = torch.stack([rg.pack_weight(ctx, t.cuda()) for t in w])
        return (lambda *args: rg.regione_linear_grouped(ctx, x.cuda(), packed, None, *args)), x.double().numpy(), w.double().numpy()
    xc, wc = rng.integers(0, 16, (m, k)).astype(np.uint8), rng.integers(0, 16, (weights, n, k)).astype(np.uint8)
    one = lambda rows: np.full((rows, k // 32), 127, np.uint8)
    packed = torch.empty(weights, rg.regione_packed_weight_mxfp4_bytes(n, k), dtype=torch.uint8, device="cuda")
    for i in range(weights):
        rg.regione_pack_weight_mxfp4(ctx, up(mx.pack_codes(wc[i])), up(one(n)), n, k, packed[i])
    q, s = up(mx.pack_codes(xc)), up(mx.scale_steps(one(m)))
    return (lambda *args: rg.regione_linear_mxfp4_grouped(ctx, q, s, packed, None, *args)), mx.values(xc, one(m)), np.stack([mx.values(c, one(n)) for c in wc])


@pytest.mark.parametrize("fmt", ["mxfp4", "bf16"])
@pytest.mark.parametrize("offsets", [[20, 40, 0, 10], [200, 333, 40, 199, 3, 40]])
def test_groups_in_any_order(ctx, fmt, offsets):
    m, n, k, weights = 340, 72, 192, len(offsets) - 1
    call, xv, wv = operands(ctx, fmt, m, n, k, weights)
    y = torch.full((m, n), UNTOUCHED, device="cuda")
    call(torch.tensor(offsets, dtype=torch.int32, device="cuda"), None, weights, weights, m, n, k, rg.ACT_NONE, rg.FP32, y)
    assert np.array_equal(y.cpu().double().numpy(), mx.grouped(xv, wv, None, offsets, None, np.full((m, n), UNTOUCHED)))


@pytest.mark.parametrize("fmt", ["mxfp4", "bf16"])
@pytest.mark.parametrize("tile", [0, 1, 9, 11, 42, 72])
@pytest.mark.parametrize("m,offsets", [(1024, [0, 1024] * 2), (300, [1, 299] * 75), (40, [39, 0, 40] * 300)])
def test_shared_rows(ctx, fmt, tile, m, offsets):
    """Every value is that of one of the groups, or what was there; nothing around the result is written."""
    n, k, weights, groups = 72, 128, 2, len(offsets) - 1
    call, xv, wv = operands(ctx, fmt, m, n, k, weights)
    flat = torch.full(((m + 2) * n,), UNTOUCHED, device="cuda")
    use = torch.tensor([i // 2 % 2 for i in range(groups)], dtype=torch.int32, device="cuda")
    rg.regione_tune_mx(ctx, tile)
    call(torch.tensor(offsets, dtype=torch.int32, device="cuda"), use, groups, weights, m, n, k, rg.ACT_NONE, rg.FP32, flat[n:-n])
    rg.regione_tune_mx(ctx, 0)
    got = flat.view(m + 2, n).cpu().double().numpy()
    assert (got[[0, -1]] == UNTOUCHED).all()
    got, (lo, hi) = got[1:-1], (min(offsets), max(offsets))
    assert ((got == xv @ wv[0].T) | (got == xv @ wv[1].T) | (got == UNTOUCHED)).all() and (got[:lo] == UNTOUCHED).all() and (got[hi:] == UNTOUCHED).all()


def test_more_shared_tiles_than_32_bits_count(ctx):
    """32768 groups of all 2^24 rows."""
    m, n, k, groups = 1 << 24, 8, 32, 65535
    q = torch.randint(0, 256, (m, k // 2), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=torch.uint8)
    s = torch.full((rg.regione_mxfp4_scale_bytes(m, k, rg.MX_SCALE_STEPS),), 127, dtype=torch.uint8, device="cuda")
    wc = np.random.default_rng(2).integers(0, 16, (n, k)).astype(np.uint8)
    w = torch.empty(rg.regione_packed_weight_mxfp4_bytes(n, k), dtype=torch.uint8, device="cuda")
    rg.regione_pack_weight_mxfp4(ctx, up(mx.pack_codes(wc)), up(np.full((n, 1), 127, np.uint8)), n, k, w)
    offsets = torch.tensor([0, m] * (groups // 2 + 1), dtype=torch.int32, device="cuda")
    y = torch.full((m + 1, n), UNTOUCHED, device="cuda")
    rg.regione_linear_mxfp4_grouped(ctx, q, s, w, None, offsets, torch.zeros(groups, dtype=torch.int32, device="cuda"), groups, 1, m, n, k, rg.ACT_NONE, rg.FP32, y)
    rows = sorted({int(r) for r in np.random.default_rng(3).integers(0, m, 4000)} | {0, m - 1})
    got = y[rows].cpu().double().numpy()
    want = mx.values(mx.unpack_codes(q[rows].cpu().numpy()), np.full((len(rows), 1), 127, np.uint8)) @ mx.values(wc, np.full((n, 1), 127, np.uint8)).T
    assert ((got == want) | (got == UNTOUCHED)).all() and (y[m] == UNTOUCHED).all()
