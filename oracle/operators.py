"""Norm, products by group, scores and distillation in fp64 numpy -- TEST INFRASTRUCTURE ONLY.

Shares nothing with the GPU library: each function is its formula, element by element where
numpy has no name for it.
"""
from __future__ import annotations

import numpy as np


def rms_norm(H, w, eps):
    """(Y, r): r = (mean of a row's squares + eps)^(-1/2), Y = H r w."""
    H = np.asarray(H, dtype=np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        r = 1.0 / np.sqrt((H * H).sum(1) / H.shape[1] + eps)
        return H * r[:, None] * w, r


def rms_norm_grad(H, r, dY, w, dH=None):
    """(dX, dw, what dX's terms add up to in magnitude, dw's likewise)."""
    H, dY = np.asarray(H, dtype=np.float64), np.asarray(dY, dtype=np.float64)
    x, u = H * r[:, None], dY * w
    dX = r[:, None] * (u - x * (u * x).mean(1, keepdims=True))
    size = np.abs(r)[:, None] * (np.abs(u) + np.abs(x) * np.abs(u * x).mean(1, keepdims=True))
    if dH is not None:
        dX, size = dX + dH, size + np.abs(dH)
    return dX, (dY * x).sum(0), size, np.abs(dY * x).sum(0)


def grouped(A, W, offsets, transpose):
    """(C, |A||W|), zeros in rows without a group."""
    A, W = np.asarray(A, dtype=np.float64), np.asarray(W, dtype=np.float64)
    C = np.zeros((A.shape[0], W.shape[1] if transpose else W.shape[2]))
    M = np.zeros_like(C)
    for g in range(W.shape[0]):
        r = slice(int(offsets[g]), int(offsets[g + 1]))
        B = W[g].T if transpose else W[g]
        C[r], M[r] = A[r] @ B, np.abs(A[r]) @ np.abs(B)
    return C, M


def grouped_grad(A, G, offsets):
    """(dW, |A|^T|G|) of each group."""
    A, G = np.asarray(A, dtype=np.float64), np.asarray(G, dtype=np.float64)
    parts = [slice(int(a), int(b)) for a, b in zip(offsets[:-1], offsets[1:])]
    return np.stack([A[r].T @ G[r] for r in parts]), np.stack([np.abs(A[r]).T @ np.abs(G[r]) for r in parts])


def log_softmax(s):
    """log p of every class; NaN in rows that have no distribution."""
    s = np.asarray(s, dtype=np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        x = s - s.max(1, keepdims=True)
        return x - np.log(np.exp(x).sum(1, keepdims=True))


def _plogp(lp):
    with np.errstate(invalid="ignore"):
        return np.where(np.exp(lp) == 0, 0.0, np.exp(lp) * lp)


def scores(s, ids):
    """(log p of the classes, entropy, log p of all)."""
    lp = log_softmax(s)
    v = lp.shape[1]
    got = np.array([0.0 if i < 0 else lp[r, i] if i < v else np.nan for r, i in enumerate(ids)])
    return got, -_plogp(lp).sum(1), lp


def best(s, k):
    """The k largest of each row: by value (NaN largest, -0 equal to 0), then the lower index."""
    s = np.asarray(s, dtype=np.float64)
    out = np.zeros((s.shape[0], k), dtype=np.int64)
    for r, row in enumerate(s):
        rank = np.where(np.isnan(row), np.inf, np.clip(row, -1e300, 1e300))
        out[r] = np.lexsort((np.arange(row.size), -rank))[:k]
    return out


def scores_grad(lp, entropy, ids, g, e):
    """Gradient of sum(g log p + e entropy) by the logits."""
    n, v = lp.shape
    p = np.exp(lp)
    d = np.zeros((n, v))
    for r in range(n):
        if g is not None and ids[r] >= 0:
            if ids[r] >= v:
                d[r] = np.nan
                continue
            d[r] -= g[r] * p[r]
            d[r, ids[r]] += g[r]
        if e is not None:
            d[r] -= e[r] * np.where(p[r] == 0, 0.0, _plogp(lp[r:r + 1])[0] + p[r] * entropy[r])
    return d


def distill(s, ids, t, temperature):
    """(loss, gradient by the logits of its sum, q, log p at the alternatives, log p of all)."""
    s, t = np.asarray(s, dtype=np.float64), np.asarray(t, dtype=np.float64)
    T = float(temperature)
    lp = log_softmax(s / T)
    n, v = s.shape
    loss, d = np.zeros(n), np.zeros((n, v))
    q, at = np.zeros(t.shape), np.zeros(t.shape)
    for r in range(n):
        on = (ids[r] >= 0) & ~(t[r] == -np.inf)
        if not on.any():
            continue
        if (ids[r][on] >= v).any():
            loss[r], d[r] = np.nan, np.nan
            continue
        with np.errstate(invalid="ignore"):
            w = np.where(on, np.exp((t[r] - t[r][on].max()) / T), 0.0)
        q[r] = w / w.sum()
        at[r] = np.where(on, lp[r, np.where(on, ids[r], 0)], 0.0)
        with np.errstate(divide="ignore", invalid="ignore"):
            loss[r] = T * T * np.where(q[r] > 0, q[r] * (np.log(q[r]) - at[r]), 0.0 * q[r]).sum()
        d[r] = T * np.exp(lp[r])
        for i, j in enumerate(ids[r]):
            if on[i]:
                d[r, j] -= T * q[r, i]
    return loss, d, q, at, lp
