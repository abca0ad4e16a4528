"""The sequence branch in float64, written from the formulas (numpy, plain loops where order matters)."""
from __future__ import annotations

import numpy as np


def embed_fwd(table, ids, scale):
    """Rows by id, scaled; zeros for ids outside [0, rows)."""
    table = np.asarray(table, np.float64)
    out = np.zeros((len(ids), table.shape[1]))
    for i, v in enumerate(np.asarray(ids)):
        if 0 <= v < table.shape[0]:
            out[i] = scale * table[v]
    return out


def embed_bwd(ids, grad, rows, scale):
    """The table's gradient, and the sum of its terms' magnitudes."""
    grad = np.asarray(grad, np.float64)
    out = np.zeros((rows, grad.shape[1]))
    size = np.zeros_like(out)
    for i, v in enumerate(np.asarray(ids)):
        if 0 <= v < rows:
            out[v] += scale * grad[i]
            size[v] += abs(scale) * np.abs(grad[i])
    return out, size


def layer_norm_fwd(x, gamma, beta, eps):
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    h = (x - mean[:, None]) * rstd[:, None]
    y = h * (1.0 if gamma is None else gamma) + (0.0 if beta is None else beta)
    return y, mean, rstd


def layer_norm_bwd(x, gamma, mean, rstd, dy):
    """dx, dgamma, dbeta."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    rstd = np.asarray(rstd, np.float64)[:, None]
    h = (x - np.asarray(mean, np.float64)[:, None]) * rstd
    g = dy * (1.0 if gamma is None else gamma)
    dx = rstd * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    return dx, (dy * h).sum(0), dy.sum(0)


def _row(x):
    """(p, log p) of one row without its masked items, and which items those are not."""
    there = x != -np.inf
    if not there.any():
        return None
    v = x[there]
    if np.isnan(v).any() or np.isposinf(v).any():
        return there, np.full(v.shape, np.nan), np.full(v.shape, np.nan)
    lp = v - v.max() - np.log(np.exp(v - v.max()).sum())
    return there, np.exp(lp), lp


def token_logprob(x, targets, k):
    """logprob, entropy, top_ids, top_logprobs."""
    x = np.asarray(x, np.float64)
    R, V = x.shape
    logprob, entropy = np.zeros(R), np.zeros(R)
    ids, lps = np.full((R, k), -1, np.int64), np.full((R, k), -np.inf)
    for r in range(R):
        aimed = 0 <= targets[r] < V
        row = _row(x[r])
        if row is None:
            logprob[r] = -np.inf if aimed else 0.0
            continue
        there, p, lp = row
        full = np.full(V, -np.inf)
        full[there] = lp
        entropy[r] = -(p * lp).sum()
        if aimed:
            logprob[r] = full[targets[r]] if not np.isnan(lp).any() else np.nan
        order = np.lexsort((np.arange(V), -x[r]))           # by falling score, then by item
        order = order[x[r][order] > -np.inf][:k]
        ids[r, :len(order)] = order
        lps[r, :len(order)] = full[order]
    return logprob, entropy, ids, lps


def token_logprob_bwd(x, targets, grad_logprob, grad_entropy):
    """dx, and the sum of its terms' magnitudes."""
    x = np.asarray(x, np.float64)
    R, V = x.shape
    dx, size = np.zeros((R, V)), np.zeros((R, V))
    for r in range(R):
        row = _row(x[r])
        if row is None:
            continue
        there, p, lp = row
        h = -(p * lp).sum()
        aimed = 0 <= targets[r] < V
        gl = grad_logprob[r] if aimed and grad_logprob is not None else 0.0
        gh = grad_entropy[r] if grad_entropy is not None else 0.0
        at = np.nonzero(there)[0]
        hot = (at == targets[r]).astype(np.float64) if aimed else np.zeros(len(at))
        dx[r, at] = gl * (hot - p) - gh * p * (lp + h)
        size[r, at] = abs(gl) * (hot + p) + abs(gh) * p * (np.abs(lp) + h)
    return dx, size


def grad_clip(grads, max_norm):
    """norm, coefficient."""
    norm = float(np.sqrt(sum(float((np.asarray(g, np.float64) ** 2).sum()) for g in grads)))
    return norm, float(np.minimum(1.0, max_norm / (norm + 1e-6)))          # (NaN stays)
