"""Products over groups of rows with weights of their own, 4-bit and bf16, against oracle/mx_reference.py in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import mx_reference as mx
from paper_2510_25590_amd import binding as rg

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return rg.Context(256, 4, 64, 1024, 64, 64)


class Operands:
    """x and weights of one format on the device, and their values; `fine` keeps float32 sums exact."""

    def __init__(self, ctx, fmt, m, n, k, weights, seed, fine):
        rng = np.random.default_rng(seed)
        self.fmt, self.m, self.n, self.k, self.weights = fmt, m, n, k, weights
        if fmt == "bf16":
            draw = (lambda *s: rng.integers(-8, 9, s) / 4.0) if fine else (lambda *s: rng.normal(size=s))
            x, w = (torch.from_numpy(draw(*s)).float().to(torch.bfloat16) for s in ((m, k), (weights, n, k)))
            self.x, self.w = x.cuda(), torch.stack([rg.pack_weight(ctx, w[i].cuda()) for i in range(weights)])
            self.xv, self.wv = x.double().numpy(), w.double().numpy()
        else:
            codes = lambda r: rng.integers(0, 16, (r, k)).astype(np.uint8)
            scale = lambda r: (127 + (0 if fine else rng.integers(-4, 5, (r, k // 32))) * np.ones((r, k // 32), int)).astype(np.uint8)
            up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
            xc, xs = codes(m), scale(m)
            self.x, self.xs, self.xv = up(mx.pack_codes(xc)), up(mx.scale_steps(xs)), mx.values(xc, xs)
            self.w = torch.empty(weights, rg.regione_packed_weight_mxfp4_bytes(n, k), dtype=torch.uint8, device="cuda")
            self.wv = np.empty((weights, n, k))
            for i in range(weights):
                wc, ws = codes(n), scale(n)
                rg.regione_pack_weight_mxfp4(ctx, up(mx.pack_codes(wc)), up(ws), n, k, self.w[i])
                self.wv[i] = mx.values(wc, ws)

    def call(self, ctx, offsets, use, bias, act, y):
        o = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        u = None if use is None else torch.tensor(use, dtype=torch.int32, device="cuda")
        b = None if bias is None else torch.from_numpy(bias).cuda()
        args = (o, u, len(offsets) - 1, self.weights, self.m, self.n, self.k, rg.ACT_GELU_TANH if act else rg.ACT_NONE, rg.FP32 if y.dtype == torch.float32 else rg.BF16, y)
        if self.fmt == "bf16":
            rg.regione_linear_grouped(ctx, self.x, self.w, b, *args)
        else:
            rg.regione_linear_mxfp4_grouped(ctx, self.x, self.xs, self.w, b, *args)
        return y


def offsets_of(sizes, first=0):
    return [first] + [int(v) for v in first + np.cumsum(sizes)]


CASES = [  # sizes of the groups, row of the first, rows in all, columns, K, weights, which
    ([1], 0, 1, 8, 64, 1, None),
    ([0, 0, 0], 0, 3, 16, 64, 3, None),
    ([3, 5], 0, 8, 40, 128, 2, None),
    ([0, 7, 0, 1, 16, 0], 2, 30, 72, 320, 6, None),
    ([17, 33, 1, 64], 0, 115, 130, 192, 4, None),
    ([100, 200, 100, 200], 0, 600, 256, 512, 2, [0, 1, 0, 1]),
    ([5] * 70, 1, 360, 64, 128, 3, [i % 3 for i in range(70)]),
    ([0] * 64 + [2] + [0] * 100 + [300], 0, 302, 96, 256, 2, [0] * 65 + [1] * 101),
    ([257, 0, 129, 515], 3, 910, 520, 1024, 4, [3, 2, 1, 0]),
    ([700], 33, 800, 264, 448, 5, [4]),
    ([40, 1100, 9], 0, 1149, 1160, 768, 3, None),
]


@pytest.mark.parametrize("fmt", ["mxfp4", "bf16"])
@pytest.mark.parametrize("sizes,first,m,n,k,weights,use", CASES)
def test_groups_exact(ctx, fmt, sizes, first, m, n, k, weights, use):
    """Products that float32 adds exactly in any order (multiples of 1/16, 4 k at most in bf16; of 1/4, 36 k at most in 4 bits); rows of no group stay as they were."""
    o = Operands(ctx, fmt, m, n, k, weights, m + n, True)
    y = o.call(ctx, offsets_of(sizes, first), use, None, False, torch.full((m, n), 0.3125, device="cuda"))
    want = mx.grouped(o.xv, o.wv, None, offsets_of(sizes, first), use, np.full((m, n), 0.3125))
    assert np.array_equal(y.cpu().double().numpy(), want)


@pytest.mark.parametrize("fmt", ["mxfp4", "bf16"])
@pytest.mark.parametrize("act,out", [(False, torch.bfloat16), (True, torch.bfloat16), (True, torch.float32)])
@pytest.mark.parametrize("sizes,first,m,n,k,weights,use", CASES)
def test_groups(ctx, fmt, act, out, sizes, first, m, n, k, weights, use):
    """The bound of tests/test_gpu_mxfp4.py: float32 sums of k products and a bias in any order, the activation's slope and rounding, the output's rounding.  In bf16 a product of two
    values has 16 bits and is exact in float32."""
    o = Operands(ctx, fmt, m, n, k, weights, m * 3 + n, False)
    bias = np.random.default_rng(1).normal(size=(weights, n)).astype(np.float32)
    got = o.call(ctx, offsets_of(sizes, first), use, bias, act, torch.full((m, n), 0.3125, dtype=out, device="cuda")).cpu().double().numpy()
    z = mx.grouped(o.xv, o.wv, bias, offsets_of(sizes, first), use, np.zeros((m, n)))
    err = (k + 1) * 2.0 ** -24 * mx.grouped(np.abs(o.xv), np.abs(o.wv), np.abs(bias), offsets_of(sizes, first), use, np.zeros((m, n)))
    want = z
    if act:
        want, err = mx.gelu_tanh(z), 1.13 * err + 2.0 ** -18 * np.abs(z)
    err = err + torch.finfo(out).eps / 2 * (np.abs(want) + err) + 2.0 ** -140
    inside = np.zeros(m, bool)
    inside[first:first + sum(sizes)] = True
    assert np.all(got[~inside] == 0.3125)
    assert not inside.any() or np.max(np.abs(got - want)[inside] / err[inside]) <= 1.0


@pytest.mark.parametrize("fmt", ["mxfp4", "bf16"])
@pytest.mark.parametrize("offsets,use", [([-5, 4, 9, 400], None), ([2, 9, 9, 30], [0, 7, -1]), ([10, 3, 20, 20], [0, 1, 2]), ([40, 50, 60, 70], None), ([0, 2 ** 31 - 1, -2 ** 31, -1], [2, 1, 0])])
def test_offsets_and_weights_outside(ctx, fmt, offsets, use):
    """Offsets are held within the rows; groups that end before they start or whose weight does not exist are left out."""
    o = Operands(ctx, fmt, 40, 48, 192, 3, 4, True)
    y = o.call(ctx, offsets, use, None, False, torch.full((40, 48), 0.3125, device="cuda"))
    want = mx.grouped(o.xv, o.wv, None, offsets, use, np.full((40, 48), 0.3125))
    assert np.array_equal(y.cpu().double().numpy(), want)


@pytest.mark.parametrize("fmt", ["mxfp4", "bf16"])
def test_rows_of_other_groups_do_not_matter(ctx, fmt):
    """What stands in rows of no group, NaN included, is not read into any result."""
    o = Operands(ctx, fmt, 96, 64, 256, 2, 6, True)
    if fmt == "bf16":
        o.x[:10], o.x[70:] = float("nan"), float("inf")
    else:
        o.xs.view(-1, 96, 8)[:, :10] = 255
        o.xs.view(-1, 96, 8)[:, 70:] = 255
    y = o.call(ctx, [10, 41, 70], None, None, False, torch.full((96, 64), 0.3125, device="cuda"))
    want = mx.grouped(o.xv, o.wv, None, [10, 41, 70], None, np.full((96, 64), 0.3125))
    assert np.array_equal(y.cpu().double().numpy(), want)


@pytest.mark.parametrize("fmt", ["mxfp4", "bf16"])
def test_one_group_is_the_plain_product(ctx, fmt):
    """The same sums, up to float32 order, as the call without groups."""
    m, n, k = 300, 384, 768
    o = Operands(ctx, fmt, m, n, k, 1, 9, True)
    y = o.call(ctx, [0, m], None, None, False, torch.empty(m, n, device="cuda"))
    z = torch.empty(m, n, device="cuda")
    if fmt == "bf16":
        rg.regione_linear(ctx, o.x, o.w[0], None, m, n, k, rg.ACT_NONE, rg.FP32, z)
    else:
        rg.regione_linear_mxfp4(ctx, o.x, o.xs, o.w[0], None, m, n, k, rg.ACT_NONE, rg.FP32, z)
    assert torch.equal(y, z)


@pytest.mark.parametrize("fmt", ["mxfp4", "bf16"])
def test_captured_and_replayed_with_other_groups(fmt):
    """A captured call reads its offsets when it runs: every replay, with eager work of the same context's stream between, gives what the offsets of then ask for."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = rg.Context(256, 4, 64, 1024, 64, 64, stream=stream)
        o = Operands(ctx, fmt, 500, 320, 1024, 3, 11, True)
        offsets = torch.tensor([0, 100, 100, 500], dtype=torch.int32, device="cuda")
        y = torch.zeros(500, 320, device="cuda")
        args = (offsets, None, 3, 3, 500, 320, 1024, rg.ACT_NONE, rg.FP32, y)
        call = lambda: rg.regione_linear_grouped(ctx, o.x, o.w, None, *args) if fmt == "bf16" else rg.regione_linear_mxfp4_grouped(ctx, o.x, o.xs, o.w, None, *args)
        call()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
        for which in ([0, 100, 100, 500], [0, 1, 400, 410], [3, 3, 490, 500], [0, 0, 0, 0]):
            offsets.copy_(torch.tensor(which, dtype=torch.int32))
            y.fill_(0.3125)
            graph.replay()
            got = y.cpu().double().numpy()
            y.fill_(0.3125)
            call()
            stream.synchronize()
            assert np.array_equal(got, mx.grouped(o.xv, o.wv, None, which, None, np.full((500, 320), 0.3125)))
            assert np.array_equal(y.cpu().double().numpy(), got)
        del graph
        ctx.close()
