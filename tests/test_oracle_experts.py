"""The 64-bit reference of routing and adapters (oracle/expert_reference.py) against hand-written results and properties that follow from the definitions."""
import numpy as np

from oracle import expert_reference as ex


def test_route_by_hand():
    l = np.array([[0.0, 2.0, 1.0, 2.0]])
    e, w = ex.route(l, None, None, "softmax", 1, 1, 1, 3, True, 1.0)
    assert e.tolist() == [[1, 3, 2]]                                     # equal logits: the lower expert first
    p = np.exp([2.0, 2.0, 1.0])
    assert np.allclose(w, p / p.sum(), rtol=1e-15)
    # a bias decides who is chosen and is no part of the weight
    e, w = ex.route(l, np.array([5.0, 0.0, 0.0, 0.0]), None, "sigmoid", 1, 1, 1, 1, False, 2.0)
    assert e.tolist() == [[0]] and np.allclose(w, 2.0 * 0.5)
    # groups {0, 1} and {2, 3}: best single value in the first, best sum in the second
    l = np.array([[3.0, -9.0, 1.0, 1.0]])
    assert ex.route(l, None, None, "sigmoid", 2, 1, 1, 1, False, 1.0)[0].tolist() == [[0]]
    assert ex.route(l, None, None, "sigmoid", 2, 1, 2, 1, False, 1.0)[0].tolist() == [[2]]


def test_route_without_choices():
    l = np.array([[-np.inf, np.nan, 0.0], [-np.inf, -np.inf, np.nan], [1.0, 2.0, 3.0]])
    e, w = ex.route(l, None, [1, 1, 0], "softmax", 1, 1, 1, 2, True, 1.0)
    assert e.tolist() == [[2, -1], [-1, -1], [-1, -1]] and w.tolist() == [[1.0, 0.0], [0.0, 0.0], [0.0, 0.0]]


def test_slots_sort_and_combine_brings_back():
    rng = np.random.default_rng(0)
    expert = rng.integers(-1, 5, (40, 3)).astype(np.int32)
    offsets, row_token, slot = ex.slots(expert, 5, np.full(120, -7))
    assert offsets[0] == 0 and offsets[-1] == (expert >= 0).sum() and np.all(row_token[offsets[-1]:] == -7)
    for g in range(5):
        mine = row_token[offsets[g]:offsets[g + 1]]
        assert np.all(np.diff(mine) >= 0) and mine.tolist() == [t for t in range(40) for j in range(3) if expert[t, j] == g]
    rows = row_token[:offsets[-1], None].astype(float) + 1.0             # every row tells its token
    out, _ = ex.combine(rows, slot, None, None)
    assert np.array_equal(out[:, 0], (np.arange(40) + 1.0) * (expert >= 0).sum(axis=1))


def test_adapters_are_low_rank_updates_of_the_weight():
    rng = np.random.default_rng(1)
    x, w, a, b = rng.normal(size=(6, 8)), rng.normal(size=(5, 8)), rng.normal(size=(3, 2, 8)), rng.normal(size=(3, 5, 2))
    which, weight = np.array([[0, 1], [2, -1], [-1, -1], [1, 1], [0, 9], [2, 0]]), rng.normal(size=(6, 2))
    y, _ = ex.adapters(x, w, None, a, b, which, weight)
    for r in range(6):
        full = w + sum(weight[r, s] * b[i] @ a[i] for s, i in enumerate(which[r]) if 0 <= i < 3)
        assert np.allclose(y[r], full @ x[r], rtol=1e-12)
