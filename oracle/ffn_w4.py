"""Expert FFN with weights of 4 bits, oracle -- TEST INFRASTRUCTURE ONLY (numpy, float64).

The expert function of oracle/ffn.py (SwiGLU) with  W[n][k] = (code[n][k] - zero[k / G][n]) * scale[k / G][n], two codes per byte, the even input
in the low four bits; without zero points the zero is 8.
"""
from __future__ import annotations

import numpy as np

from .ffn import _silu


def unpack(q, scale, zero=None):
    """q uint8 [n][k/2], scale float64 [k/G][n], zero uint8 [k/G][n] or None -> float64 [n][k]"""
    n, half = q.shape
    group = 2 * half // scale.shape[0]
    w = np.empty((n, 2 * half))
    for k in range(2 * half):
        code = (q[:, k // 2] >> (4 * (k % 2))) & 15
        z = 8.0 if zero is None else (zero[k // group] & 15).astype(np.float64)
        w[:, k] = (code.astype(np.float64) - z) * scale[k // group]
    return w


def expert_ffn(x, expert_of_row, weights):
    """x float64 [M][d]; expert_of_row int [M], negative = no row; weights: per expert (gate, up, down) of unpack() ->
    (y [M][d], what the arithmetic adds up to in absolute values: dict of h, g, u and their sums)."""
    M, d = x.shape
    y = np.zeros((M, d))
    h_all = [None] * len(weights)
    for e, (wg, wu, wd) in enumerate(weights):
        sel = np.flatnonzero(expert_of_row == e)
        if sel.size == 0:
            continue
        g, u = x[sel] @ wg.T, x[sel] @ wu.T
        h = _silu(g) * u
        y[sel] = h @ wd.T
        h_all[e] = (sel, g, u, h)
    return y, h_all
