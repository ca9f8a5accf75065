"""GPU parity of the microscaled 4-bit rows and products with oracle/mx_reference.py: codes, scales and values bit for bit, products within the rounding of float32 sums."""
import numpy as np
import pytest
import torch

from oracle import mx_reference as mx
from paper_2510_25590_amd import binding as rg

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return rg.Context(256, 4, 64, 1024, 64, 64)


def up(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def rows_of(rng, rows, cols, dtype):
    """Rows with what a quantiser meets: a wide range in a block, zeros, ties, values at both ends of the type, subnormal numbers; as the type holds them, in float64."""
    x = rng.normal(size=(rows, cols)) * np.exp2(rng.integers(-6, 4, (rows, cols)))
    x[rng.random((rows, cols)) < 0.05] = 0.0
    for r, f in ((1, 0.0), (2, 2.0 ** 120), (3, 2.0 ** -126), (4, 2.0 ** -133), (5, 2.0 ** -148)):
        if rows > r:
            x[r] *= f
    if rows > 6:
        x[6] = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.0, -0.25], cols) * np.repeat(np.exp2(rng.integers(-30, 30, cols // 32)), 32)
    t = torch.from_numpy(x).to(dtype)
    if dtype == torch.bfloat16:     # the conversion from float64 goes by way of float32
        t = torch.from_numpy(x).float().to(dtype)
    return t


def quantized(ctx, x, layout):
    q, s = rg.quantize_rows_mxfp4(ctx, x, layout)
    return q.cpu().numpy(), s.cpu().numpy()


@pytest.mark.parametrize("rows,cols", [(1, 32), (8, 64), (7, 256), (9, 288), (33, 1024), (130, 3072), (5, 12288), (1025, 544), (3, 32 * 4099)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_bit_exact(ctx, rows, cols, dtype):
    x = rows_of(np.random.default_rng(rows * 7 + cols), rows, cols, dtype)
    codes, scale = mx.quantize(x.double().numpy())
    q, s = quantized(ctx, x.cuda(), rg.MX_SCALE_ROWS)
    assert np.array_equal(s.reshape(scale.shape), scale)
    assert np.array_equal(q, mx.pack_codes(codes))
    q, s = quantized(ctx, x.cuda(), rg.MX_SCALE_STEPS)
    want = mx.scale_steps(scale)
    assert np.array_equal(q, mx.pack_codes(codes))
    assert np.array_equal(s.reshape(want.shape)[:, :rows], want[:, :rows])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_blocks_with_nan_and_infinity(ctx, dtype):
    x = torch.randn(6, 320, generator=torch.Generator().manual_seed(1)).to(dtype)
    x[0, 5], x[1, 40], x[2, 319], x[3, 100], x[4] = float("nan"), float("inf"), float("-inf"), torch.finfo(dtype).max, torch.finfo(dtype).tiny
    codes, scale = mx.quantize(x.double().numpy())
    assert (scale == 255).sum() == 3
    q, s = quantized(ctx, x.cuda(), rg.MX_SCALE_ROWS)
    assert np.array_equal(s.reshape(scale.shape), scale) and np.array_equal(q, mx.pack_codes(codes))
    y = torch.empty(6, 320, dtype=torch.float32, device="cuda")
    rg.regione_dequantize_rows_mxfp4(ctx, up(q), up(s), rg.MX_SCALE_ROWS, 6, 320, rg.FP32, y)
    assert np.array_equal(y.cpu().double().numpy(), mx.values(codes, scale), equal_nan=True)


@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", [rg.MX_SCALE_ROWS, rg.MX_SCALE_STEPS])
def test_dequantize_every_code_under_every_scale(ctx, out, layout):
    """All 16 codes under all scales whose values fit both types, and NaN."""
    scale = np.concatenate([np.arange(253), [255]]).astype(np.uint8).reshape(2, 127)
    codes = np.tile(np.arange(16, dtype=np.uint8), (2, 127 * 2))
    y = torch.empty(codes.shape, dtype=out, device="cuda")
    s = scale if layout == rg.MX_SCALE_ROWS else mx.scale_steps(scale)
    rg.regione_dequantize_rows_mxfp4(ctx, up(mx.pack_codes(codes)), up(s), layout, *codes.shape, rg.FP32 if out == torch.float32 else rg.BF16, y)
    assert np.array_equal(y.cpu().double().numpy(), mx.values(codes, scale), equal_nan=True)


@pytest.mark.parametrize("rows,cols", [(1, 32), (820, 3072), (8704, 288), (65, 4128)])
def test_round_trip_and_rows_behind_the_last(ctx, rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, cols, generator=g, device="cuda").to(torch.bfloat16)
    q = torch.full((rows + 1, cols // 2), 77, dtype=torch.uint8, device="cuda")
    n = rg.regione_mxfp4_scale_bytes(rows, cols, rg.MX_SCALE_STEPS)
    s = torch.full((n + 64,), 77, dtype=torch.uint8, device="cuda")
    y = torch.full((rows + 1, cols), 77.0, dtype=torch.bfloat16, device="cuda")
    rg.regione_quantize_rows_mxfp4(ctx, x, rg.BF16, rows, cols, rg.MX_SCALE_STEPS, q, s)
    rg.regione_dequantize_rows_mxfp4(ctx, q, s, rg.MX_SCALE_STEPS, rows, cols, rg.BF16, y)
    assert (q[rows] == 77).all() and (s[n:] == 77).all() and (y[rows] == 77.0).all()
    codes, scale = mx.quantize(x.double().cpu().numpy())
    assert np.array_equal(y[:rows].cpu().double().numpy(), mx.values(codes, scale))


def weight(ctx, codes, scale):
    n, k = codes.shape
    out = torch.empty(rg.regione_packed_weight_mxfp4_bytes(n, k), dtype=torch.uint8, device="cuda")
    rg.regione_pack_weight_mxfp4(ctx, up(mx.pack_codes(codes)), up(scale), n, k, out)
    return out


def random_operand(rng, rows, k, spread):
    codes = rng.integers(0, 16, (rows, k)).astype(np.uint8)
    scale = (127 + rng.integers(-spread, spread + 1, (rows, k // 32))).astype(np.uint8)
    return codes, scale


def linear(ctx, xc, xs, wc, ws, bias, act, out, y=None):
    m, k = xc.shape
    n = len(wc)
    y = torch.full((m, n), 9.0, dtype=out, device="cuda") if y is None else y
    rg.regione_linear_mxfp4(ctx, up(mx.pack_codes(xc)), up(mx.scale_steps(xs)), weight(ctx, wc, ws), None if bias is None else up(bias), m, n, k,
                            rg.ACT_GELU_TANH if act else rg.ACT_NONE, rg.FP32 if out == torch.float32 else rg.BF16, y)
    return y.cpu().double().numpy()


def check(got, xv, wv, bias, act, out):
    """Any order of float32 additions of k exact products and a bias is off by at most (k + 1) 2^-24 sum |products|.  The activation passes errors on with a slope of at most 1.13; its own: the
    exponential's argument, below 16 in magnitude where its result matters, carries a few roundings of 2^-24 and the exponential, the reciprocal and their products a few more, so
    that the result is off by less than 2^-18 of |z|.  Then the rounding to the output's type."""
    z = xv @ wv.T + (0.0 if bias is None else bias.astype(np.float64))
    err = (xv.shape[1] + 1) * 2.0 ** -24 * (np.abs(xv) @ np.abs(wv).T + (0.0 if bias is None else np.abs(bias)))
    want = z
    if act:
        want, err = mx.gelu_tanh(z), 1.13 * err + 2.0 ** -18 * np.abs(z)
    err = err + torch.finfo(out).eps / 2 * (np.abs(want) + err) + 2.0 ** -140
    worst = np.max(np.abs(got - want) / err)
    assert worst <= 1.0, worst


SHAPES = [(1, 1, 32), (1, 64, 256), (2, 33, 64), (15, 40, 96), (16, 96, 512), (17, 7, 288), (33, 129, 1056), (36, 768, 256), (64, 256, 3072), (100, 1000, 544), (128, 264, 2048), (129, 513, 320),
          (257, 512, 1024), (300, 2304, 768), (820, 1152, 1536), (1000, 130, 15360), (1382, 3072, 3072), (2049, 264, 224)]


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_products_exact(ctx, m, n, k):
    """Scales of one: every sum is a multiple of 1/4 below 36 k <= 2^20, which float32 holds exactly in any order."""
    rng = np.random.default_rng(m + n + k)
    xc, xs = random_operand(rng, m, k, 0)
    wc, ws = random_operand(rng, n, k, 0)
    got = linear(ctx, xc, xs, wc, ws, None, False, torch.float32)
    assert np.array_equal(got, mx.values(xc, xs) @ mx.values(wc, ws).T)


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act", [False, True])
def test_products(ctx, m, n, k, out, act):
    rng = np.random.default_rng(m * n + k)
    xc, xs = random_operand(rng, m, k, 6)
    wc, ws = random_operand(rng, n, k, 6)
    ws = (ws - 6).astype(np.uint8)
    bias = rng.normal(size=n).astype(np.float32) if n % 2 else None
    check(linear(ctx, xc, xs, wc, ws, bias, act, out), mx.values(xc, xs), mx.values(wc, ws), bias, act, out)


@pytest.mark.parametrize("m,n,k", [(3, 64, 96), (200, 300, 800), (700, 256, 288)])
def test_scales_at_the_ends_and_nan(ctx, m, n, k):
    """Factors that meet in the middle of the range: 2^-127 by 2^+119 and the other way round, and one block of NaN in a row and in a column."""
    rng = np.random.default_rng(5)
    xc, xs = random_operand(rng, m, k, 0)
    wc, ws = random_operand(rng, n, k, 0)
    low = rng.random(k // 32) < 0.5
    xs[:, low], ws[:, low] = 0, 246
    xs[:, ~low], ws[:, ~low] = 246, 0
    xs[m - 1, 1], ws[n // 2, 0] = 255, 255
    got = linear(ctx, xc, xs, wc, ws, None, False, torch.float32)
    want = mx.values(xc, xs) @ np.nan_to_num(mx.values(wc, ws)).T
    nan = np.zeros((m, n), bool)
    nan[m - 1], nan[:, n // 2] = True, True
    assert np.array_equal(np.isnan(got), nan)
    assert np.array_equal(got[~nan], want[~nan])


@pytest.mark.parametrize("n,offset", [(64, 0), (64, 1), (72, 3), (67, 0)])
def test_results_out_of_alignment_and_nothing_around_them(ctx, n, offset):
    m, k = 37, 320
    rng = np.random.default_rng(n + offset)
    xc, xs = random_operand(rng, m, k, 1)
    wc, ws = random_operand(rng, n, k, 1)
    flat = torch.full((m * n + 64,), 5.0, dtype=torch.bfloat16, device="cuda")
    y = flat[offset:offset + m * n].view(m, n)
    got = linear(ctx, xc, xs, wc, ws, None, False, torch.bfloat16, y)
    check(got, mx.values(xc, xs), mx.values(wc, ws), None, False, torch.bfloat16)
    assert (flat[:offset] == 5.0).all() and (flat[offset + m * n:] == 5.0).all()


def test_padding_rows_of_the_scales_are_not_read_into_results(ctx):
    """An odd number of rows: the scale bytes of the row that fills it up may be anything."""
    m, n, k = 5, 40, 512
    rng = np.random.default_rng(8)
    xc, xs = random_operand(rng, m, k, 2)
    wc, ws = random_operand(rng, n, k, 2)
    steps = mx.scale_steps(xs)
    steps[:, m] = 255
    y = torch.empty(m, n, dtype=torch.float32, device="cuda")
    rg.regione_linear_mxfp4(ctx, up(mx.pack_codes(xc)), up(steps), weight(ctx, wc, ws), None, m, n, k, rg.ACT_NONE, rg.FP32, y)
    check(y.cpu().double().numpy(), mx.values(xc, xs), mx.values(wc, ws), None, False, torch.float32)


def test_a_chain_as_it_is_used(ctx):
    """Rows quantised, multiplied with quantised weights, activated, quantised again and multiplied: each stage on the library's own input of it."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(205, 768, generator=g, device="cuda").to(torch.bfloat16)
    w1, w2 = (0.05 * torch.randn(s, generator=g, device="cuda") for s in ((1024, 768), (768, 1024)))
    b1 = 0.1 * torch.randn(1024, generator=g, device="cuda")
    p1, p2 = rg.pack_weight_mxfp4(ctx, w1), rg.pack_weight_mxfp4(ctx, w2.to(torch.bfloat16))
    q, s = rg.quantize_rows_mxfp4(ctx, x)
    h = torch.empty(205, 1024, dtype=torch.bfloat16, device="cuda")
    rg.regione_linear_mxfp4(ctx, q, s, p1, b1, 205, 1024, 768, rg.ACT_GELU_TANH, rg.BF16, h)
    q2, s2 = rg.quantize_rows_mxfp4(ctx, h)
    y = torch.empty(205, 768, dtype=torch.float32, device="cuda")
    rg.regione_linear_mxfp4(ctx, q2, s2, p2, None, 205, 768, 1024, rg.ACT_NONE, rg.FP32, y)
    v = lambda t: mx.values(*mx.quantize(t.double().cpu().numpy()))
    check(h.cpu().double().numpy(), v(x), v(w1), b1.cpu().numpy(), True, torch.bfloat16)
    check(y.cpu().double().numpy(), v(h), v(w2.to(torch.bfloat16)), None, False, torch.float32)
