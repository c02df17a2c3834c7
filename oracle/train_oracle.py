"""Plain CPU fp64 oracle of the operators beside the compressed linear layer.  TEST INFRASTRUCTURE ONLY.

8-bit checkpoints of activations, the linear layer and the gated activation that keep one, and the vocabulary's product with its
softmax cross entropy.  numpy on float64, unblocked, from the definitions in include/acc.h; no code is shared with the library.
"""
from __future__ import annotations

import numpy as np

BLOCK = 32
LIMIT = {"e4m3": 448.0, "int8": 127.0}
TOP = 1.875 * 2.0 ** 127


def _e4m3_values():
    """Value of each of the 256 e4m3 codes (sign, four bits of exponent with bias 7, three bits of mantissa)."""
    code = np.arange(256)
    expo, mant = (code >> 3) & 15, code & 7
    v = np.where(expo == 0, mant * 2.0 ** -9, (1 + mant / 8.0) * 2.0 ** (expo - 7.0))
    v = np.where((code & 0x7F) == 0x7F, np.nan, v)
    return np.where(code & 0x80, -v, v)


def _int8_values():
    v = np.arange(256, dtype=np.int64)
    v = np.where(v > 127, v - 256, v).astype(np.float64)
    v[0x80] = np.nan
    return v


VALUES = {"e4m3": _e4m3_values(), "int8": _int8_values()}


def _nearest_code(y, fmt):
    """Code of the nearest value, ties to the even one.  |y| <= LIMIT."""
    if fmt == "int8":
        return np.rint(y).astype(np.int64) & 0xFF
    grid = VALUES["e4m3"][:0x7F]                       # the positive finite values, increasing
    mag = np.abs(y)
    hi = np.clip(np.searchsorted(grid, mag), 0, 0x7E)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - mag, mag - grid[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return code | (np.signbit(y).astype(np.int64) << 7)


def act8_pack(X, fmt):
    """X [n, c] -> (Q uint8 [n, c], E uint8 [ceil(n / 32), c])."""
    X = np.asarray(X, dtype=np.float64)
    n, c = X.shape
    fine = np.isfinite(X)
    kept = np.clip(np.where(fine, X, 0.0), -TOP, TOP)
    blocks = -(-n // BLOCK)
    e = np.full((blocks, c), -100, dtype=np.int64)
    for b in range(blocks):
        big = np.abs(kept[b * BLOCK:(b + 1) * BLOCK]).max(axis=0)
        while np.any(big > LIMIT[fmt] * 2.0 ** e[b].astype(np.float64)):
            e[b] += big > LIMIT[fmt] * 2.0 ** e[b].astype(np.float64)
    y = kept / 2.0 ** np.repeat(e, BLOCK, axis=0)[:n].astype(np.float64)
    q = np.where(fine, _nearest_code(y, fmt), 0x7F if fmt == "e4m3" else 0x80)
    return q.astype(np.uint8), (e + 127).astype(np.uint8)


def act8_unpack(Q, E, fmt):
    n = Q.shape[0]
    return VALUES[fmt][Q] * 2.0 ** (np.repeat(E.astype(np.float64), BLOCK, axis=0)[:n] - 127)


def gated(G, U):
    return G / (1 + np.exp(-G)) * U


def gated_bwd(dH, G, U):
    s = 1 / (1 + np.exp(-G))
    return dH * U * s * (1 + G * (1 - s)), dH * G * s


def linear_ce(X, W, targets):
    """Losses and log-sum-exp per token of the logits X . W^T, W [v, d]; negative targets have loss 0."""
    z = X @ W.T
    top = z.max(axis=1, keepdims=True)
    lse = (np.log(np.exp(z - top).sum(axis=1, keepdims=True)) + top)[:, 0]
    keep = targets >= 0
    zt = z[np.arange(len(z)), np.where(keep, targets, 0)]
    return np.where(keep, lse - zt, 0.0), lse


def linear_ce_bwd(X, W, targets, dloss):
    """Gradients of sum(dloss * loss): dX and dW."""
    z = X @ W.T
    p = np.exp(z - z.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    keep = targets >= 0
    p[np.arange(len(z)), np.where(keep, targets, 0)] -= 1.0
    dz = np.where(keep, dloss, 0.0)[:, None] * p
    dz[~keep] = 0.0
    return dz @ W, dz.T @ X
