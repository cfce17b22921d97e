"""Router oracle -- TEST INFRASTRUCTURE ONLY (numpy, float64).

Section 2.1 of the paper: the router picks topk experts per token; their weights are the scores of the chosen experts (softmax over all
experts or the sigmoid of each logit), divided by their sum if renormalised.  One token at a time, one slot at a time; -inf and NaN
are masked experts, which have a score of zero and are never chosen (-1 where none is left).
"""
from __future__ import annotations

import numpy as np


def _scores(row, score):
    there = ~(np.isnan(row) | np.isneginf(row))
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            return np.where(there, 1.0 / (1.0 + np.exp(-np.where(there, row, 0.0))), 0.0)
    p = np.zeros(len(row))
    if there.any():
        top = row[there].max()
        with np.errstate(invalid="ignore"):
            e = np.where(there, np.where(row == top, 1.0, np.exp(np.where(there, row, 0.0) - top)), 0.0)
        p = np.where(there, e, 0.0) / e[there].sum()
    return p


def choose(row, topk):
    """Largest first, the lower index first among equal ones."""
    left = [e for e in range(len(row)) if not (np.isnan(row[e]) or np.isneginf(row[e]))]
    ids = []
    for _ in range(topk):
        if not left:
            ids.append(-1)
            continue
        best = left[0]
        for e in left[1:]:
            if row[e] > row[best]:
                best = e
        ids.append(best)
        left.remove(best)
    return ids


def topk(logits, k, score, renormalise, scale=1.0):
    T = logits.shape[0]
    ids, gates = np.full((T, k), -1, dtype=np.int32), np.zeros((T, k))
    for t in range(T):
        ids[t] = choose(logits[t], k)
        gates[t] = weights(logits[t], ids[t], score, renormalise, scale)
    return ids, gates


def weights(row, ids, score, renormalise, scale=1.0):
    """Weights of the slots of one token for given ids; slots out of range and masked experts have the weight zero."""
    s = _scores(row, score)
    w = np.array([s[i] if 0 <= i < len(row) else 0.0 for i in ids])
    if renormalise and w.sum() > 0:
        w = w / w.sum()
    return scale * w


def topk_backward(d_gates, logits, ids, score, renormalise, scale=1.0):
    """d_logits = (Jacobian of the weights)^T d_gates, the Jacobian built one slot and one expert at a time."""
    T, E = logits.shape
    out = np.zeros((T, E))
    for t in range(T):
        s = _scores(logits[t], score)
        there = ~(np.isnan(logits[t]) | np.isneginf(logits[t]))
        # ds[i][e] = d score_i / d logit_e
        ds = np.diag(s * (1.0 - s)) if score == "sigmoid" else np.diag(s) - np.outer(s, s)
        slots = [j for j in range(ids.shape[1]) if 0 <= ids[t, j] < E and there[ids[t, j]]]
        total = sum(s[ids[t, j]] for j in slots)
        for j in slots:
            i = ids[t, j]
            if not renormalise:
                out[t] += scale * d_gates[t, j] * ds[i]
            elif total > 0:
                out[t] += scale * d_gates[t, j] * (ds[i] / total - s[i] / total ** 2 * sum(ds[ids[t, k]] for k in slots))
        out[t] = np.where(there, out[t], 0.0)
    return out
