"""Weights are formed in 64 bits and rounded once: half a step of float32 (2^-24), and 2^-44 relative for what comes before."""
import numpy as np
import pytest
import torch

from paper_2510_25590_amd import binding as rg
from route_util import check_repeated
from test_gpu_experts import route, up

pytestmark = pytest.mark.gpu
ONCE = 2.0 ** -24 * (1 + 2.0 ** -20)


@pytest.fixture(scope="module")
def ctx():
    return rg.Context(256, 4, 64, 1024, 64, 64)


def test_renormalised_weights_next_to_a_power_of_two(ctx):
    """Weights 1 / (1 + a + b) a little above a half, where half a step is 2^-24 of the value and an exponential that is off by 2^-32 shows; a is exp of about -ln(2) / 2, the hardest for a series around
    multiples of ln(2)."""
    rng = np.random.default_rng(0)
    n = 1 << 18
    a = (-0.3465 + 0.001 * rng.random(n)).astype(np.float32)
    total = 2.0 / (1.0 + 0.001 * rng.random(n))
    b = np.log(total - 1.0 - np.exp(a.astype(np.float64))).astype(np.float32)
    l = np.stack([a, np.zeros(n, np.float32), b], axis=1)
    expert, weight = route(ctx, up(l), None, None, "softmax", 1, 1, 1, 3, True, 1.0)
    assert (expert == [1, 0, 2]).all()
    p = np.exp(l[:, [1, 0, 2]].astype(np.float64))
    want = p / p.sum(axis=1, keepdims=True)
    assert np.max(np.abs(weight - want) / want) <= ONCE


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens", [300, 2047, 2048, 4099])
@pytest.mark.parametrize("experts", [7, 64, 128, 200, 256, 1000])
def test_softmax_over_all_experts(ctx, experts, tokens, dtype):
    """... not renormalised, without bias and groups: the sum over all experts in 64 bits too."""
    rng = np.random.default_rng(experts + tokens)
    logits = up(1.5 * rng.normal(size=(tokens, experts)), torch.float32).to(dtype)
    k = min(experts, 8)
    expert, weight = route(ctx, logits, None, None, "softmax", 1, 1, 1, k, False, 2.5)
    l = logits.cpu().double().numpy()
    assert np.array_equal(expert, np.argsort(-l, axis=1, kind="stable")[:, :k])
    p = np.exp(l - l.max(axis=1, keepdims=True))
    want = 2.5 * np.take_along_axis(p / p.sum(axis=1, keepdims=True), expert.astype(np.int64), axis=1)
    assert np.max(np.abs(weight - want) / want) <= ONCE


@pytest.mark.parametrize("tokens", [7, 2047, 2048, 4099])
@pytest.mark.parametrize("k", [1, 3, 8])
def test_renormalised_sigmoids_far_below_one(ctx, k, tokens):
    """Scores of 1e-300 and less, whose reciprocals pass 2^1000; they count as 0 from e^-709 on.  Two exponentials of arguments of hundreds are off by 2^-44 together, and a quarter more for what is behind them."""
    l = np.full((7, 8), -720.0, np.float32)
    l[0] = -690.0 - 0.1 * np.arange(8)
    l[1] = -693.0 - 0.25 * np.arange(8)
    l[2] = -700.0 + 0.3 * np.arange(8)
    l[3] = -708.96875 + 0.03125 * np.arange(8)
    l[4, :3] = -709.0, -708.5, -709.03125
    l[5, 5] = -650.0
    check_repeated(ctx, up(l), tokens, None, "sigmoid", 1, 1, 1, k, True, 1.0, weight=2.0 ** -24 * (1 + 2.0 ** -19))
