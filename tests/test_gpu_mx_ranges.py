"""4-bit and grouped products where float32 ends: subnormal sums, the activation over its whole range; groups with long K; a context whose stream is not the current one."""
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


def four_bit(ctx, rng, m, n, k, x_byte=127, w_byte=127, weights=1):
    """Rows, scales, packed weights and the values of both, all under one scale byte each."""
    xc, wc = rng.integers(0, 16, (m, k)).astype(np.uint8), rng.integers(0, 16, (weights, n, k)).astype(np.uint8)
    xs, ws = np.full((m, k // 32), x_byte, np.uint8), np.full((n, k // 32), w_byte, np.uint8)
    packed = torch.empty(weights, rg.regione_packed_weight_mxfp4_bytes(n, k), dtype=torch.uint8, device="cuda")
    for i in range(weights):
        rg.regione_pack_weight_mxfp4(ctx, up(mx.pack_codes(wc[i])), up(ws), n, k, packed[i])
    return up(mx.pack_codes(xc)), up(mx.scale_steps(xs)), packed, mx.values(xc, xs), np.stack([mx.values(c, ws) for c in wc])


def bf16(ctx, rng, m, n, k, unit=0.25, weights=1):
    """Rows, packed weights and the values of both: whole multiples of `unit`, eight at most."""
    x, w = (torch.from_numpy(rng.integers(-8, 9, s) * unit).float().to(torch.bfloat16) for s in ((m, k), (weights, n, k)))
    return x.cuda(), torch.stack([rg.pack_weight(ctx, t.cuda()) for t in w]), x.double().numpy(), w.double().numpy()


@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("splits", [1, 3])
def test_subnormal_sums_of_4_bit_products(ctx, tile, splits):
    """Multiples of 2^-149 below 36 * 4 * 800 of them: float32 holds every sum exactly, and it is subnormal."""
    m, n, k = 70, 136, 800
    x, s, w, xv, wv = four_bit(ctx, np.random.default_rng(tile), m, n, k, 0, 107)
    want = xv @ wv[0].T
    assert 0 < np.abs(want).max() < 2.0 ** -126
    rg.regione_tune_mx(ctx, tile, splits)
    for out in (torch.float32, torch.bfloat16):
        y = torch.full((m, n), 9.0, dtype=out, device="cuda")
        rg.regione_linear_mxfp4(ctx, x, s, w[0], None, m, n, k, rg.ACT_NONE, rg.FP32 if out == torch.float32 else rg.BF16, y)
        assert torch.equal(y.cpu(), torch.from_numpy(want).float().to(out))


@pytest.mark.parametrize("tile", TILES)
def test_subnormal_sums_of_groups_in_bf16(ctx, tile):
    """Multiples of 2^-146, exact as above."""
    m, n, k = 70, 136, 832
    x, w, xv, wv = bf16(ctx, np.random.default_rng(tile), m, n, k, 2.0 ** -73, 2)
    offsets = [0, 33, m]
    want = mx.grouped(xv, wv, None, offsets, None, np.zeros((m, n)))
    assert 0 < np.abs(want).max() < 2.0 ** -126
    rg.regione_tune_mx(ctx, tile)
    y = torch.full((m, n), 9.0, device="cuda")
    rg.regione_linear_grouped(ctx, x, w, None, torch.tensor(offsets, dtype=torch.int32, device="cuda"), None, 2, 2, m, n, k, rg.ACT_NONE, rg.FP32, y)
    assert np.array_equal(y.cpu().double().numpy(), want)


@pytest.mark.parametrize("fmt", ["mxfp4", "bf16"])
@pytest.mark.parametrize("tile,splits", [(1, 1), (9, 1), (11, 1), (42, 1), (72, 1), (22, 2)])
def test_activation_over_the_whole_range(ctx, fmt, tile, splits):
    """Rows of zeros, so that the bias is what the activation gets.  Its exponent, -2u log2(e) with u = sqrt(2/pi) (x + 0.044715 x^3), carries four roundings of 2^-24 (of a constant, the square, the
    sum and the product), so the exponential is off by 8 |u| 2^-24; the exponential and the reciprocal may be off by 2^-23 of their own, the divisor and the product by 2^-24.  Where the exponential
    overflows the result is zero.  A quarter of a subnormal x may be off by half a step, which the reciprocal doubles, and the product by another half."""
    special = [0.0, -0.0, np.inf, np.nan, 1e-30, -1e-30, 1e19, -1e19, 3e38, -3e38, 13.0, -13.0, -14.5, 1.5e-38, -1.5e-38, 1e-40, -3e-45]
    near = np.linspace(-13.05, -12.9, 64)
    b = np.concatenate([np.array(special), near, np.linspace(-16, 16, 512 - len(special) - len(near))]).astype(np.float32)
    m, n, k = 3, len(b), 1024
    y = torch.zeros((m, n), device="cuda")
    rg.regione_tune_mx(ctx, tile, splits)
    if fmt == "mxfp4":
        _, s, w, _, _ = four_bit(ctx, np.random.default_rng(1), m, n, k)
        rg.regione_linear_mxfp4(ctx, torch.zeros((m, k // 2), dtype=torch.uint8, device="cuda"), s, w[0], up(b), m, n, k, rg.ACT_GELU_TANH, rg.FP32, y)
    else:
        _, w, _, _ = bf16(ctx, np.random.default_rng(1), m, n, k)
        rg.regione_linear_grouped(ctx, torch.zeros((m, k), dtype=torch.bfloat16, device="cuda"), w, up(b), torch.tensor([0, m], dtype=torch.int32, device="cuda"), None, 1, 1, m, n, k,
                                  rg.ACT_GELU_TANH, rg.FP32, y)
    got, v = y.cpu().double().numpy(), b.astype(np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        u = np.sqrt(2 / np.pi) * (v + 0.044715 * v ** 3)
        want = v / (1 + np.exp(-2 * u))
    want[np.isposinf(v)] = np.inf
    assert np.array_equal(got[0], got[1], equal_nan=True) and np.array_equal(got[0], got[2], equal_nan=True)
    assert np.array_equal(np.isnan(got[0]), np.isnan(v)) and np.array_equal(np.isposinf(got[0]), np.isposinf(v))
    ok = np.isfinite(v)
    overflow = -2 * u[ok] * np.log2(np.e) >= 128 * (1 - 2.0 ** -20)
    bound = np.abs(want[ok]) * (8 * np.minimum(np.abs(u[ok]), 50) + 6) * 2.0 ** -24 + np.abs(want[ok]) * overflow + 1.5 * 2.0 ** -149
    assert np.all(np.abs(got[0][ok] - want[ok]) <= bound)


@pytest.mark.parametrize("fmt", ["mxfp4", "bf16"])
@pytest.mark.parametrize("tile", [0, 1, 9, 11, 31, 42, 72])
@pytest.mark.parametrize("sizes,n,k", [([512, 0, 820], 264, 12288), ([17, 300, 1, 65], 136, 4096), ([3, 40, 9, 2], 72, 2112)])
def test_groups_with_long_k(ctx, fmt, tile, sizes, n, k):
    """Sums that float32 holds exactly: multiples of 1/4 below 36 k < 2^19 in 4 bits, of 1/16 below 4 k < 2^16 in bf16."""
    offsets = [0] + [int(v) for v in np.cumsum(sizes)]
    m, groups = offsets[-1], len(sizes)
    y = torch.full((m, n), 0.3125, device="cuda")
    args = (None, torch.tensor(offsets, dtype=torch.int32, device="cuda"), None, groups, groups, m, n, k, rg.ACT_NONE, rg.FP32, y)
    rg.regione_tune_mx(ctx, tile)
    if fmt == "mxfp4":
        x, s, w, xv, wv = four_bit(ctx, np.random.default_rng(k), m, n, k, weights=groups)
        rg.regione_linear_mxfp4_grouped(ctx, x, s, w, *args)
    else:
        x, w, xv, wv = bf16(ctx, np.random.default_rng(k), m, n, k, weights=groups)
        rg.regione_linear_grouped(ctx, x, w, *args)
    assert np.array_equal(y.cpu().double().numpy(), mx.grouped(xv, wv, None, offsets, None, np.zeros((m, n))))


def test_a_context_whose_stream_is_not_the_current_one():
    """The calls run on the context's stream, behind what is queued there."""
    side = torch.cuda.Stream()
    ctx = rg.Context(256, 4, 64, 1024, 64, 64, stream=side)
    m, n, k = 130, 264, 2048
    x, s, w, xv, wv = four_bit(ctx, np.random.default_rng(4), m, n, k)
    late = torch.zeros_like(x)
    y, o = torch.full((m, n), 9.0, device="cuda"), torch.tensor([0, m], dtype=torch.int32, device="cuda")
    z = torch.full((m, n), 9.0, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        busy = torch.ones(2048, 2048, device="cuda")
        for _ in range(20):
            busy = (busy @ busy).clamp_(-1.0, 1.0)
        late.copy_(x)
    rg.regione_linear_mxfp4(ctx, late, s, w[0], None, m, n, k, rg.ACT_NONE, rg.FP32, y)
    rg.regione_linear_mxfp4_grouped(ctx, late, s, w, None, o, None, 1, 1, m, n, k, rg.ACT_NONE, rg.FP32, z)
    side.synchronize()
    want = xv @ wv[0].T
    assert np.array_equal(y.cpu().double().numpy(), want) and np.array_equal(z.cpu().double().numpy(), want)
    ctx.close()
