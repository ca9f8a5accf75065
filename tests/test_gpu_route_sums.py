"""Sums of a softmax where float32 loses what counts."""
import numpy as np
import pytest

from paper_2510_25590_amd import binding as rg
from route_util import check_repeated
from test_gpu_experts import up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return rg.Context(256, 4, 64, 1024, 64, 64)


@pytest.mark.parametrize("k", [1, 2, 3])
def test_a_sum_that_rounds_up_thirty_times(ctx, k):
    """Expert 0 has a score of nearly 1, thirty others of its lane 1.03 * 2^-24 each: added to 1 one by one in float32, each counts twice.  Its score is 30 * 0.97 * 2^-24 too small then, and with a bias of
    -1 it stands behind experts 100 and 200, whose values are their biases and lie further apart than 2^-20; in truth it is the first."""
    l = np.full((1, 1023), -60.0, np.float32)
    l[0, 0] = 0.0
    l[0, 1:31] = np.log(1.03 * 2.0 ** -24)
    bias = np.full(1023, -5.0, np.float32)
    bias[[0, 100, 200]] = -1.0, -2.2e-6, -3.2e-6
    check_repeated(ctx, up(l), 5, bias, "softmax", 33, 33, 1, k, False, 1.0)
