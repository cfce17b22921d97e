"""Norms around a MoE block, oracle -- TEST INFRASTRUCTURE ONLY (numpy, float64).

Section 2.1 of the paper: a MoE block replaces the feed-forward block of a transformer layer, which stands between residual
connections.  With rms(v) = sqrt(mean(v^2) + eps) over a token's columns:

    norm:  out = x / rms(x) * weight
    join:  u = z / rms(z) * post_weight (or z);  out = scale * stream + gate * u;  next = out / rms(out) * next_weight

The gradients are the chain rule with the Jacobian of v / rms(v), J[i][j] = (delta_ij - n_i n_j / d) / rms, n = v / rms (which is symmetric).
"""
from __future__ import annotations

import numpy as np


def _rms(v, eps):
    return np.sqrt((v * v).mean(axis=-1, keepdims=True) + eps)


def norm(x, weight, eps):
    return x / _rms(x, eps) * weight


def join(z, stream, post_weight, gate, next_weight, scale, eps):
    u = z if post_weight is None else norm(z, post_weight, eps)
    if gate is not None:
        u = gate[:, None] * u
    out = scale * stream + u
    return out, None if next_weight is None else norm(out, next_weight, eps)


def norm_gradient(d_out, x, weight, eps):
    """(gradient of x, gradient of weight)"""
    r = _rms(x, eps)
    n = x / r
    dn = d_out * weight
    return (dn - n * (dn * n).mean(axis=-1, keepdims=True)) / r, (d_out * n).sum(axis=0)


def join_backward(d_out, d_next, z, out, post_weight, gate, next_weight, scale, eps):
    """Gradients of join's inputs from those of out (None = zero) and next; out as the forward pass returned it."""
    total = np.zeros_like(out) if d_out is None else d_out.copy()
    g = dict(d_gate=None, d_post_weight=None, d_next_weight=None)
    if next_weight is not None:
        through, g["d_next_weight"] = norm_gradient(d_next, out, next_weight, eps)
        total = total + through
    g["d_stream"] = scale * total
    u = z if post_weight is None else norm(z, post_weight, eps)
    du = total
    if gate is not None:
        g["d_gate"] = (total * u).sum(axis=1)
        du = gate[:, None] * total
    if post_weight is None:
        g["d_z"] = du
    else:
        g["d_z"], g["d_post_weight"] = norm_gradient(du, z, post_weight, eps)
    return g
