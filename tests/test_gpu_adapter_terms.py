"""What the terms that an adapter's inner products are kept in have to hold: sums of more bits than two bf16 numbers have, next to results that cancel the largest of them."""
import numpy as np
import pytest
import torch

from paper_2510_25590_amd import binding as rg
from test_gpu_adapters import TILES, up

pytestmark = pytest.mark.gpu
BITS = 23


class Powers:
    """Inner products that are any whole numbers of 23 bits: x holds bits, rank r of A the powers of two from r on (cyclic).  Column c of B has a single 1, at rank c % rank, so that its share is one inner
    product; W takes away the bits from 2^keep on.  Every sum on the way is a whole number below 2^24: exact in float32 in any order, results below 2^keep whole and, up to eight bits, exact in bf16."""
    def __init__(self, ctx, m, n, k, rank, count, keep, seed):
        rng = np.random.default_rng(seed)
        bits = rng.integers(0, 2, (m, BITS))
        x = np.zeros((m, k))
        x[:, :BITS] = bits
        power = 2.0 ** ((np.arange(BITS)[None, :] + np.arange(rank)[:, None]) % BITS)       # [rank, bit]
        a = np.zeros((rank, k))
        a[:, :BITS] = power
        b = np.zeros((n, rank))
        b[np.arange(n), np.arange(n) % rank] = 1.0
        w = np.zeros((n, k))
        w[:, :BITS] = np.where(power >= 2.0 ** keep, -power, 0.0)[np.arange(n) % rank]
        self.m, self.n, self.k, self.rank, self.count = m, n, k, rank, count
        bf = lambda v: up(v, torch.bfloat16)
        self.x, self.wp = bf(x), rg.pack_weight(ctx, bf(w))
        self.ap = rg.pack_adapters(ctx, bf(np.stack([a] * count)), bf(np.stack([b] * count)))
        self.which = up(rng.integers(0, count, (m, 1)).astype(np.int32))
        self.want = bits @ (np.where(power < 2.0 ** keep, power, 0.0)[np.arange(n) % rank]).T

    def check(self, ctx, out):
        y = torch.full((self.m, self.n), 7.0, dtype=out, device="cuda")
        rg.regione_linear_adapters(ctx, self.x, self.wp, None, self.ap, self.which, None, self.count, 1, self.rank, self.m, self.n, self.k, rg.ACT_NONE, rg.FP32 if out == torch.float32 else rg.BF16, y)
        assert np.array_equal(y.cpu().double().numpy(), self.want)


@pytest.fixture(scope="module")
def ctx():
    return rg.Context(256, 4, 64, 1024, 64, 64)


SHAPES = [(1, 64, 64), (7, 200, 128), (16, 64, 64), (45, 2048, 64), (300, 520, 192), (3000, 64, 64), (1100, 1032, 320)]


@pytest.mark.parametrize("rank", [1, 16, 23, 32, 40, 64, 100])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_float32_results_have_all_bits(ctx, m, n, k, rank):
    """W takes nothing away: 23 bits of every inner product, ranks of one to seven blocks of 16."""
    Powers(ctx, m, n, k, rank, 3, BITS, m + rank).check(ctx, torch.float32)


@pytest.mark.parametrize("splits", [1, 2])
@pytest.mark.parametrize("tile", TILES)
def test_float32_results_of_every_tile(tile, splits):
    ctx = rg.Context(256, 4, 64, 1024, 64, 64)
    rg.regione_tune_gemm(ctx, tile, splits)
    for rank, count, k in ((9, 3, 64), (20, 2, 320), (48, 2, 128)):
        Powers(ctx, 270, 260, k, rank, count, BITS, tile + rank).check(ctx, torch.float32)
    ctx.close()


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rank", [1, 16, 23, 40, 64])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_results_that_cancel_the_largest_terms(ctx, m, n, k, rank, out):
    """W takes away all but the lowest eight bits: what is left is all that a result has."""
    Powers(ctx, m, n, k, rank, 3, 8, m + rank + 1).check(ctx, out)


@pytest.mark.parametrize("splits", [1, 2])
@pytest.mark.parametrize("tile", TILES)
def test_cancelled_bf16_results_of_every_tile(tile, splits):
    ctx = rg.Context(256, 4, 64, 1024, 64, 64)
    rg.regione_tune_gemm(ctx, tile, splits)
    for rank, count, k in ((9, 3, 64), (20, 2, 320), (48, 2, 128)):
        Powers(ctx, 270, 260, k, rank, count, 8, tile + rank).check(ctx, torch.bfloat16)
    ctx.close()


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n", [(3, 64), (45, 2048), (300, 520), (3000, 64)])
def test_inner_products_above_the_largest_bf16(ctx, m, n, out):
    """2^128 - 2^118: finite in float32, rounded to bf16 infinite.  B holds 2^-100 in the first column and zeros in the others."""
    k, rank = 64, 5
    x, a, b = np.zeros((m, k)), np.zeros((rank, k)), np.zeros((n, rank))
    x[:, :3] = 1.0
    a[2, :3] = 2.0 ** 128 - 2.0 ** 120, 2.0 ** 119, 2.0 ** 118
    b[0, 2] = 2.0 ** -100
    x[1] *= -1.0
    total = float(a[2].sum())
    assert float(np.float32(total)) == total < 2.0 ** 128 and np.isinf(torch.tensor(total, dtype=torch.float32).to(torch.bfloat16).item())
    bf = lambda v: up(v, torch.bfloat16)
    ap = rg.pack_adapters(ctx, bf(a[None]), bf(b[None]))
    wp = rg.pack_weight(ctx, torch.zeros(n, k, dtype=torch.bfloat16, device="cuda"))
    y = torch.full((m, n), 7.0, dtype=out, device="cuda")
    rg.regione_linear_adapters(ctx, bf(x), wp, None, ap, torch.zeros(m, 1, dtype=torch.int32, device="cuda"), None, 1, 1, rank, m, n, k, rg.ACT_NONE, rg.FP32 if out == torch.float32 else rg.BF16, y)
    want = np.zeros((m, n))
    want[:, 0] = total * 2.0 ** -100 * x[:, 0]
    assert torch.equal(y.cpu(), torch.from_numpy(want).to(out))
