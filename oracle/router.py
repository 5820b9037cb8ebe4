"""The router in front of the expert layer (oracle; test infrastructure only).

Scores are softmax(l) or sigmoid(l) over a token's E logits.  The k experts are those of the largest
logits, or with a bias of the largest score + bias; ties go to the lower index; an expert whose key is
-inf or NaN is never chosen (-1 in its place).  Weights are scale * score, or scale * score / (sum of the
chosen scores).  Everything in float64.
"""

import numpy as np


def scores(logits, score):
    z = np.asarray(logits, dtype=np.float64)
    with np.errstate(all="ignore"):
        if score == "sigmoid":
            return 1.0 / (1.0 + np.exp(-z))
        m = z.max(axis=1, keepdims=True)
        e = np.exp(z - np.where(m == -np.inf, 0.0, m))
        total = e.sum(axis=1, keepdims=True)
        return e / np.where(total == 0.0, 1.0, total)


def choose(logits, bias, k, score):
    """topk_idx [T, k]."""
    z = np.asarray(logits, dtype=np.float64)
    key = z.copy() if bias is None else scores(z, score) + np.asarray(bias, dtype=np.float64)
    key[~(z > -np.inf)] = -np.inf
    key[np.isnan(key)] = -np.inf
    idx = np.argsort(-key, axis=1, kind="stable")[:, :k]
    chosen = np.take_along_axis(key, idx, axis=1)
    return np.where(chosen == -np.inf, -1, idx)


def log_scores(logits, score):
    """Logarithms of the scores, up to a constant of the row for softmax."""
    z = np.asarray(logits, dtype=np.float64)
    if score == "softmax":
        return z
    with np.errstate(all="ignore"):
        return np.minimum(z, 0.0) - np.log1p(np.exp(-np.abs(z)))


def weights(logits, idx, score, normalize, scale):
    """Routing weights [T, k] of chosen experts."""
    idx = np.asarray(idx)
    at = np.maximum(idx, 0)
    kept = idx >= 0
    if not normalize:
        p = np.take_along_axis(scores(logits, score), at, axis=1)
    else:
        v = np.where(kept, np.take_along_axis(log_scores(logits, score), at, axis=1), -np.inf)
        p = scores(v, "softmax")
    return np.where(kept, scale * p, 0.0)


def weights_bwd(logits, idx, dprobs, score, normalize, scale):
    """Gradient of sum(dprobs * weights) with respect to the logits [T, E]."""
    z = np.asarray(logits, dtype=np.float64)
    idx = np.asarray(idx)
    kept = idx >= 0
    at = np.maximum(idx, 0)
    dp = np.where(kept, np.asarray(dprobs, dtype=np.float64), 0.0)
    out = np.zeros_like(z)
    s = scores(z, score)
    zj = np.take_along_axis(z, at, axis=1)
    with np.errstate(all="ignore"):
        one_minus = 1.0 / (1.0 + np.exp(zj)) if score == "sigmoid" else np.ones_like(zj)
    if normalize:
        r = weights(z, idx, score, True, 1.0)
        g = scale * one_minus * r * (dp - (r * dp).sum(axis=1, keepdims=True))
    else:
        sj = np.where(kept, np.take_along_axis(s, at, axis=1), 0.0)
        g = scale * sj * dp * one_minus
    for j in range(idx.shape[1]):
        rows = np.nonzero(kept[:, j])[0]
        np.add.at(out, (rows, at[rows, j]), g[rows, j])
    if not normalize and score == "softmax":
        out -= s * g.sum(axis=1, keepdims=True)
    return out
