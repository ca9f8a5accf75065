"""CPU oracle for the microscaled 4-bit (MXFP4) variant of the dense projections and for products over groups of rows.

TEST INFRASTRUCTURE ONLY (see regione_oracle.py): the product never imports this file and this file imports nothing
from the product.

The paper (arXiv 2510.25590) does not use 4-bit arithmetic; what is computed is fixed by the public OCP microscaling
specification (E2M1 elements, one E8M0 scale per 32 consecutive values): the exponent of a block is that of its largest
magnitude less E2M1's largest exponent, 2; elements are rounded to nearest, ties to the even code, and saturate; a block
with a NaN or an infinity has the NaN scale.  A block of zeros has the smallest scale (the specification leaves it open).
Values are float64, in which every product of two E2M1 values and two scales is exact.

Parity pins: tests/test_oracle_mx.py.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK, STEP = 32, 256
VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def e2m1_encode(t) -> np.ndarray:
    """Codes (bit 3 the sign) of float64 values."""
    t = np.asarray(t, dtype=np.float64)
    a = np.abs(t)
    # half a step below 2, one from 2 to 4, two from 4 on
    step = np.where(a < 2.0, 0.5, np.where(a < 4.0, 1.0, 2.0))
    v = np.minimum(np.rint(a / step) * step, 6.0)
    return np.searchsorted(VALUES, v).astype(np.uint8) | (np.signbit(t).astype(np.uint8) << 3)


def quantize(x) -> tuple[np.ndarray, np.ndarray]:
    """x [rows, cols] -> codes [rows, cols] (one per entry) and scale bytes [rows, cols / 32]."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    b = x.reshape(rows, cols // BLOCK, BLOCK)
    bad = ~np.isfinite(b).all(axis=2)
    amax = np.where(bad, 1.0, np.abs(np.where(np.isfinite(b), b, 0.0)).max(axis=2))
    e = np.where(amax > 0, np.frexp(amax)[1] - 3, -127)
    e = np.clip(e, -127, 127)
    codes = e2m1_encode(np.where(bad[:, :, None], 0.0, b) * np.ldexp(1.0, -e)[:, :, None])
    return codes.reshape(rows, cols), np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, scale) -> np.ndarray:
    """Float64 values of codes [rows, cols] and scale bytes [rows, cols / 32]; NaN under a scale of 255."""
    codes = np.asarray(codes, dtype=np.int64)
    v = VALUES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.ldexp(1.0, np.asarray(scale, dtype=np.int64) - 127)
    s = np.where(np.asarray(scale) == 255, np.nan, s)
    return v * np.repeat(s, BLOCK, axis=1)


def pack_codes(codes) -> np.ndarray:
    """Two codes per byte, the lower column in the lower bits."""
    c = np.asarray(codes, dtype=np.uint8)
    return c[:, 0::2] | (c[:, 1::2] << 4)


def unpack_codes(q) -> np.ndarray:
    q = np.asarray(q, dtype=np.uint8)
    return np.stack((q & 15, q >> 4), axis=2).reshape(q.shape[0], -1)


def scale_steps(scale) -> np.ndarray:
    """Scale bytes [rows, blocks] in the layout of steps: [steps, rows rounded up to even, 8], block b of a step at byte 4 (b % 2) + b / 2.  Bytes of rows that
    do not exist are zero here and may be anything."""
    rows, blocks = np.asarray(scale).shape
    steps = -(-blocks // 8)
    out = np.zeros((steps, (rows + 1) // 2 * 2, 8), dtype=np.uint8)
    for b in range(blocks):
        out[b // 8, :rows, 4 * (b % 2) + b % 8 // 2] = scale[:, b]
    return out


def gelu_tanh(x) -> np.ndarray:
    return 0.5 * x * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3)))


def grouped(x, weights, biases, offsets, use, y) -> np.ndarray:
    """y with rows [offsets[g], offsets[g + 1]) replaced by x W^T + b of weight use[g]; x and weights are values."""
    y = np.array(y, dtype=np.float64)
    m = len(x)
    for g in range(len(offsets) - 1):
        lo, hi = (min(max(int(o), 0), m) for o in offsets[g:g + 2])
        w = g if use is None else int(use[g])
        if hi > lo and 0 <= w < len(weights):
            y[lo:hi] = x[lo:hi] @ weights[w].T + (0.0 if biases is None else biases[w])
    return y
