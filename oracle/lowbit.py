"""The microscaled formats in fp64 numpy -- TEST INFRASTRUCTURE ONLY.

Shares nothing with the GPU library.  Blocks of 32 consecutive columns of a row
(the last one may be short) share a scale byte E, which stands for 2^(E - 127);
E = 255 marks a block with a NaN or an infinity, whose values are all NaN.

``save8`` is the 8-bit form of activations: with m the block's largest magnitude
and 2^p <= m < 2^(p+1), the step is 2^(p-7) under a ReLU (unsigned codes) and
2^(p-6) otherwise, at least 2^-126; a code is the nearest whole number of steps,
ties to even, clamped to 255 (127 and -127), and under a ReLU at least 1 where
the input is not <= 0.

``quant4`` is MXFP4: the scale is 2^(p-2), at least 2^-127, an element the
nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 scales, ties to the even code, 6 beyond.
"""
from __future__ import annotations

import numpy as np

BLOCK = 32
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _scales(x, below, least):
    """(E, 2^(E-127)) per block; E = 255 and NaN for blocks that are not finite."""
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    E = np.zeros((rows, nb), dtype=np.int64)
    for b in range(nb):
        blk = x[:, b * BLOCK:(b + 1) * BLOCK]
        for r in range(rows):
            v = blk[r]
            if not np.all(np.isfinite(v)):
                E[r, b] = 255
                continue
            m = float(np.max(np.abs(v)))
            p = np.frexp(m)[1] - 1 if m > 0 else -10_000
            E[r, b] = max(p - below, least) + 127
    with np.errstate(over="ignore"):
        s = np.where(E == 255, np.nan, np.ldexp(1.0, (E - 127).astype(np.int32)))
    return E, s


def _spread(s, cols):
    return np.repeat(s, BLOCK, axis=1)[:, :cols]


def save8(P, relu: bool):
    """(codes int64, E, values, h, on) of fp64 P; on: where the ReLU's gradient is 1."""
    P = np.asarray(P, dtype=np.float64)
    on = ~(P <= 0)
    h = np.where(on, P, 0.0) if relu else P
    E, s = _scales(h, 7 if relu else 6, -126)
    S = _spread(s, P.shape[1])
    with np.errstate(invalid="ignore"):
        q = np.rint(h / S)  # (numpy rounds ties to even)
    q = np.where(np.isnan(S), 0.0, q)
    q = np.where(on, np.clip(q, 1, 255), 0.0) if relu else np.clip(q, -127, 127)
    return q.astype(np.int64), E, q * S, h, on


def quant4(X):
    """(codes 0..15, E, values) of fp64 X, blocks along the rows."""
    X = np.asarray(X, dtype=np.float64)
    E, s = _scales(X, 2, -127)
    S = _spread(s, X.shape[1])
    with np.errstate(invalid="ignore"):
        y = np.abs(X) / S
    y = np.where(np.isnan(S), 0.0, y)
    code = np.zeros(X.shape, dtype=np.int64)
    for i in range(1, 8):
        mid = 0.5 * (E2M1[i - 1] + E2M1[i])
        code = np.where((y > mid) | ((y == mid) & (i % 2 == 0)), i, code)
    values = np.where(np.signbit(X), -1.0, 1.0) * E2M1[code] * S
    return np.where(np.isnan(S), 0, code + 8 * np.signbit(X)), E, values
