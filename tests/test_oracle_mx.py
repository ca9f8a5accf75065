"""Pins of the 4-bit oracle (oracle/mx_reference.py) against the format's definition and plain arithmetic."""
import numpy as np
import pytest

from oracle import mx_reference as mx


def test_codes_by_search_over_the_format():
    rng = np.random.default_rng(1)
    mids = (mx.VALUES[:-1] + mx.VALUES[1:]) / 2
    t = np.concatenate([mids, -mids, mids * (1 + 2.0 ** -40), mids * (1 - 2.0 ** -40), rng.uniform(-8, 8, 4000), [0.0, -0.0, 7.99, -7.99, 6.0, 1e-30]])
    got = mx.e2m1_encode(t)
    for v, c in zip(t, got):
        d = np.abs(mx.VALUES - min(abs(v), 6.0))
        near = np.flatnonzero(d == d.min())
        want = near[0] if len(near) == 1 else [n for n in near if n % 2 == 0][0]
        assert c == want | (8 if np.signbit(v) else 0), v


def test_every_code_and_scale_comes_back():
    codes = np.tile(np.arange(16, dtype=np.uint8), 2)[None, :].repeat(253, axis=0)       # each block holds a 6, so the scale is fixed
    scale = np.arange(253, dtype=np.uint8)[:, None]
    c, s = mx.quantize(mx.values(codes, scale))
    assert np.array_equal(s, scale)
    assert np.array_equal(c, codes)
    assert np.array_equal(mx.unpack_codes(mx.pack_codes(codes)), codes)


@pytest.mark.parametrize("power", [-140, -128, -20, 0, 30, 120])
def test_the_error_of_a_block(power):
    """Below saturation an element is off by at most half a step of its scale: 2^e / 4 under 2 * 2^e, 2^e from 4 * 2^e on; saturated ones, of (6, 8) 2^e, by less than 2 * 2^e."""
    x = np.random.default_rng(2).normal(size=(50, 64)) * 2.0 ** power
    c, s = mx.quantize(x)
    unit = np.repeat(np.ldexp(1.0, s.astype(int) - 127), mx.BLOCK, axis=1)
    err = np.abs(mx.values(c, s) - x) / unit
    a = np.abs(x) / unit
    assert np.all(a < 8)
    assert np.all(err <= np.where(a <= 2, 0.25, np.where(a <= 4, 0.5, np.where(a <= 6, 1.0, 2.0))))
    full = s > 0
    assert np.all(np.abs(x).reshape(50, 2, 32).max(axis=2)[full] >= 4 * np.ldexp(1.0, s.astype(int) - 127)[full])


def test_special_blocks():
    x = np.zeros((1, 128))
    x[0, 40], x[0, 70] = np.nan, -np.inf
    x[0, 100] = -2.0 ** -149
    c, s = mx.quantize(x)
    assert s.tolist() == [[0, 255, 255, 0]] and c[0, 100] == 8 and not c[0, :100].any()
    v = mx.values(c, s)
    assert np.isnan(v[0, 32:96]).all() and not v[0, :32].any() and not v[0, 96:].any()


@pytest.mark.parametrize("rows,blocks", [(1, 1), (3, 8), (2, 9), (5, 20)])
def test_step_layout(rows, blocks):
    scale = np.random.default_rng(3).integers(1, 255, (rows, blocks)).astype(np.uint8)
    flat = mx.scale_steps(scale).reshape(-1)
    padded = rows + rows % 2
    assert len(flat) == -(-blocks // 8) * padded * 8
    for r in range(rows):
        for b in range(blocks):
            assert flat[(b // 8 * padded + r) * 8 + 4 * (b % 2) + b % 8 // 2] == scale[r, b]


def test_groups_by_hand():
    x, w = np.arange(12.0).reshape(6, 2), np.array([[[1.0, 0.0]], [[0.0, 2.0]]])
    y = mx.grouped(x, w, np.array([[10.0], [20.0]]), [1, 3, 3, 9], [1, 0, 0], np.full((6, 1), -1.0))
    assert y[:, 0].tolist() == [-1.0, 2 * 3 + 20.0, 2 * 5 + 20.0, 16.0, 18.0, 20.0]
    y = mx.grouped(x, w, None, [0, 2, 1, 4], [0, 1, 5], np.full((6, 1), -1.0))
    assert y[:, 0].tolist() == [0.0, 2.0, -1.0, -1.0, -1.0, -1.0]
