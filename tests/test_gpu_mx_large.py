"""4-bit rows, weights and results whose offsets pass 32 bits: sampled rows against the values that codes and scales stand for, in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import mx_reference as mx
from paper_2510_25590_amd import binding as rg

pytestmark = pytest.mark.gpu


@pytest.fixture
def ctx():
    c = rg.Context(256, 4, 64, 1024, 64, 64)
    yield c
    c.close()


def operand(rows, k, seed):
    """Random codes with scales of one, made on the device: every sum of k products is a multiple of 1/4 below 36 k, exact in float32 for k <= 2^16."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, 256, (rows, k // 2), generator=g, device="cuda", dtype=torch.uint8)


def values(q):
    codes = mx.unpack_codes(q.cpu().numpy())
    return mx.values(codes, np.full((len(codes), codes.shape[1] // 32), 127, np.uint8))


def weight(ctx, q):
    n, k = q.shape[0], 2 * q.shape[1]
    w = torch.empty(rg.regione_packed_weight_mxfp4_bytes(n, k), dtype=torch.uint8, device="cuda")
    rg.regione_pack_weight_mxfp4(ctx, q, torch.full((n, k // 32), 127, dtype=torch.uint8, device="cuda"), n, k, w)
    return w


def sample(m, row_bytes):
    """The first and last rows and those around every 2^31 bytes."""
    edges = [0, m - 1] + [e // row_bytes + d for e in range(2 ** 31, m * row_bytes, 2 ** 31) for d in (-1, 0, 1)]
    return sorted({min(max(r, 0), m - 1) for r in edges})


@pytest.mark.parametrize("m,n,k", [(300001, 136, 16384), (70001, 32768, 256), (140001, 16640, 512)])
def test_rows_and_results(ctx, m, n, k):
    q, wq = operand(m, k, 1), operand(n, k, 2)
    s = torch.full((rg.regione_mxfp4_scale_bytes(m, k, rg.MX_SCALE_STEPS),), 127, dtype=torch.uint8, device="cuda")
    y = torch.empty(m, n, dtype=torch.float32, device="cuda")
    rg.regione_linear_mxfp4(ctx, q, s, weight(ctx, wq), None, m, n, k, rg.ACT_NONE, rg.FP32, y)
    rows = sorted(set(sample(m, k // 2)) | set(sample(m, 4 * n)))
    assert np.array_equal(y[rows].cpu().double().numpy(), values(q[rows]) @ values(wq).T)


def test_weights_of_groups(ctx):
    """The last weight lies past 2^31 bytes."""
    n, k, weights = 2048, 16384, 130
    wq = [operand(n, k, 3 + i) for i in range(2)]
    packed = [weight(ctx, w) for w in wq]
    w = torch.cat([packed[i % 2] for i in range(weights)])
    assert w.numel() > 2 ** 31
    sizes = [3 if i in (0, 7, weights - 2, weights - 1) else 0 for i in range(weights)]
    offsets = np.concatenate([[0], np.cumsum(sizes)])
    m = int(offsets[-1])
    q = operand(m, k, 9)
    s = torch.full((rg.regione_mxfp4_scale_bytes(m, k, rg.MX_SCALE_STEPS),), 127, dtype=torch.uint8, device="cuda")
    y = torch.empty(m, n, dtype=torch.float32, device="cuda")
    rg.regione_linear_mxfp4_grouped(ctx, q, s, w, None, torch.tensor(offsets, dtype=torch.int32, device="cuda"), None, weights, weights, m, n, k, rg.ACT_NONE, rg.FP32, y)
    xv, wv = values(q), [values(t) for t in wq]
    for g in range(weights):
        a, b = offsets[g], offsets[g + 1]
        if b > a:
            assert np.array_equal(y[a:b].cpu().double().numpy(), xv[a:b] @ wv[g % 2].T)


@pytest.mark.parametrize("dtype,code", [(torch.bfloat16, rg.BF16), (torch.float32, rg.FP32)])
def test_quantise_and_back(ctx, dtype, code):
    rows, cols = 140001, 32800
    x = torch.empty(rows, cols, dtype=dtype, device="cuda")
    x.normal_(generator=torch.Generator(device="cuda").manual_seed(4))
    q, s = rg.quantize_rows_mxfp4(ctx, x, rg.MX_SCALE_STEPS)
    which = sample(rows, cols * x.element_size())
    codes, scale = mx.quantize(x[which].double().cpu().numpy())
    got = q.view(rows, cols // 2)[which].cpu().numpy()
    assert np.array_equal(got, mx.pack_codes(codes))
    rg.regione_dequantize_rows_mxfp4(ctx, q, s, rg.MX_SCALE_STEPS, rows, cols, code, x)
    assert np.array_equal(x[which].cpu().double().numpy(), mx.values(codes, scale))
