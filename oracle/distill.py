"""Largest logits of each row, and the distillation loss from them, in float64.

The logit of an output y is factor y, or factor silent where that is -infinity
(then it passes no gradient).
"""

import numpy as np


def logits(y, factor, silent):
    z = factor * np.asarray(y, np.float64)
    none = z == -np.inf
    return np.where(none, factor * silent, z), none


def top_logits(y, K, factor=1.0, silent=-np.inf):
    """Values and classes of the K largest of each row; equal ones by ascending class, NaN first."""
    z, _ = logits(y, factor, silent)
    order = np.argsort(np.where(np.isnan(z), -np.inf, -z) - np.where(np.isnan(z), 1.0, 0.0), axis=1, kind="stable")
    nan_first = np.stack([np.concatenate([o[np.isnan(r[o])], o[~np.isnan(r[o])]]) for o, r in zip(order, z)])
    index = nan_first[:, :K]
    return np.take_along_axis(z, index, 1), index


def distill(y, top, index, factor=1.0, silent=-np.inf, teacher_factor=1.0, weight=1.0, row_weight=None):
    """(loss, row losses, gradient with respect to y)."""
    z, none = logits(y, factor, silent)
    R, C = z.shape
    w = np.full(R, 1.0 / R) if row_weight is None else np.asarray(row_weight, np.float64)
    rows, g = np.zeros(R), np.zeros((R, C))
    for r in range(R):
        v = teacher_factor * np.asarray(top[r], np.float64)
        used = [k for k in range(len(v)) if 0 <= index[r][k] < C and v[k] != -np.inf]
        if not used or w[r] == 0 or np.all(z[r] == -np.inf):
            continue
        at = np.asarray(index[r])[used]
        log_p = v[used] - v[used].max()
        log_p = log_p - np.log(np.exp(log_p).sum())
        log_q = z[r] - z[r].max()
        log_q = log_q - np.log(np.exp(log_q).sum())
        p = np.exp(log_p)
        rows[r] = sum(pk * (lp - log_q[i]) for pk, lp, i in zip(p, log_p, at) if pk != 0)
        d = np.exp(log_q)
        np.subtract.at(d, at, p)
        g[r] = np.where(none[r], 0.0, weight * w[r] * factor * d)
    return weight * np.sum(np.where(w != 0, w * rows, 0.0)), rows, g
