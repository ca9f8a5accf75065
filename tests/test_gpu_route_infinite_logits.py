"""Logits of +infinity, which count as the largest float32, beside values that only 64 bits tell apart."""
import numpy as np
import pytest

from paper_2510_25590_amd import binding as rg
from route_util import check_repeated
from test_gpu_experts import up

pytestmark = pytest.mark.gpu
INF, MOST = np.inf, np.float32(3.4028234663852886e38)


@pytest.fixture(scope="module")
def ctx():
    return rg.Context(256, 4, 64, 1024, 64, 64)


def near_biases(e):
    """Biases of which 1 and 2 are neighbours in float32, that of 0 is the lowest; the others fall."""
    bias = (-0.5 - 0.01 * np.arange(e)).astype(np.float32)
    bias[:4] = -2.0, 0.3, np.nextafter(np.float32(0.3), np.float32(1.0)), 0.1
    return bias


def rows_of(e):
    """One infinity, two of them, an infinity and the largest value, the infinity where the near tie is, and no infinity at all."""
    l = np.zeros((6, e), np.float32)
    l[0, 0] = INF
    l[1, [0, 3]] = INF
    l[2, 0], l[2, 3] = MOST, INF
    l[3, [1, 2]] = INF
    l[4, 2] = INF
    l[5] = np.linspace(-1.0, 1.0, e)
    return l


def test_one_infinity_beside_neighbouring_biases(ctx):
    """Scores 1, 0, 0, 0 and these biases: the values are -1, 0.3, the next float32 and 0.1."""
    from test_gpu_experts import route
    expert, weight = route(ctx, up(rows_of(4)[:1]), up(near_biases(4)), None, "softmax", 1, 1, 1, 2, False, 1.0)
    assert expert.tolist() == [[2, 1]] and weight.tolist() == [[0.0, 0.0]]


@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 5, 6, 37, 8191, 8192, 8195])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts,groups,top_groups,k", [(4, 1, 1, 2), (4, 1, 1, 4), (24, 1, 1, 3), (24, 2, 2, 6), (24, 2, 1, 3), (128, 1, 1, 8), (256, 8, 4, 14), (256, 8, 4, 15)])
def test_infinite_logits_beside_near_ties(ctx, experts, groups, top_groups, k, score, tokens):
    for renorm in (False, True):
        check_repeated(ctx, up(rows_of(experts)), tokens, near_biases(experts), score, groups, top_groups, 1, k, renorm, 1.0)
