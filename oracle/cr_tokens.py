"""Token layers in 64 bits: embedding, root-mean-square norm, log probabilities, distillation (NumPy).

Written from the formulas; shares no code with the library.
"""
from __future__ import annotations

import numpy as np


def embedding(ids, table, scale=1.0):
    ids = np.asarray(ids)
    y = np.zeros(ids.shape + (table.shape[1],))
    named = (ids >= 0) & (ids < table.shape[0])
    y[named] = scale * np.asarray(table, np.float64)[ids[named]]
    return y


def embedding_backward(ids, dy, vocab, scale=1.0, padding=-1):
    """(dtable, sum of the terms' sizes) of ids [partitions, tokens], dy [partitions, tokens, width]."""
    ids, dy = np.asarray(ids), np.asarray(dy, np.float64)
    d = np.zeros((ids.shape[0], vocab, dy.shape[-1]))
    size = np.zeros_like(d)
    for p in range(ids.shape[0]):
        named = (ids[p] >= 0) & (ids[p] < vocab) & (ids[p] != padding)
        np.add.at(d[p], ids[p][named], dy[p][named])
        np.add.at(size[p], ids[p][named], np.abs(dy[p][named]))
    return scale * d, abs(scale) * size


def rms_norm(x, residual, gamma, eps):
    """(y, h, rstd)."""
    h = np.asarray(x, np.float64) + (0.0 if residual is None else np.asarray(residual, np.float64))
    rstd = 1 / np.sqrt((h * h).mean(-1) + eps)
    y = h * rstd[..., None] * (1.0 if gamma is None else np.asarray(gamma, np.float64))
    return y, h, rstd


def rms_norm_backward(dy, h, gamma, rstd, dh=None, partitions=1):
    """(dx, dgamma, sum of the terms' sizes of dgamma); rstd is the forward pass's."""
    dy, h, rstd = np.asarray(dy, np.float64), np.asarray(h, np.float64), np.asarray(rstd, np.float64)[..., None]
    xhat = h * rstd
    g = dy * (1.0 if gamma is None else np.asarray(gamma, np.float64))
    dx = rstd * (g - xhat * (g * xhat).mean(-1, keepdims=True))
    if dh is not None:
        dx = dx + np.asarray(dh, np.float64)
    terms = (dy * xhat).reshape(partitions, -1, h.shape[-1])
    return dx, terms.sum(1), np.abs(terms).sum(1)


def log_p(x, temperature=1.0):
    """(log p, m, log_sum) of rows of logits; a row of -infinity has log p = -infinity."""
    x = np.asarray(x, np.float64)
    m = x.max(-1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        z = (x - np.where(np.isinf(m), 0.0, m)) / temperature
        log_sum = np.log(np.exp(z).sum(-1, keepdims=True))
        lp = z - log_sum
    return np.where(m == -np.inf, -np.inf, lp), m[..., 0], log_sum[..., 0]


def token_log_probs(x, ids, temperature=1.0, top=0):
    """(logp, m, log_sum, entropy, top ids, top log p)."""
    lp, m, log_sum = log_p(x, temperature)
    rows, vocab = lp.shape
    with np.errstate(invalid="ignore", over="ignore"):
        p = np.exp(lp)
        entropy = -np.where(p == 0, 0.0, p * np.where(p == 0, 0.0, lp)).sum(-1)
    ids = np.asarray(ids)
    named = (ids >= 0) & (ids < vocab)
    logp = np.where(named, lp[np.arange(rows), np.where(named, ids, 0)], 0.0)
    order = np.argsort(-np.asarray(x, np.float64), axis=-1, kind="stable")[:, :top]
    return logp, m, log_sum, entropy, order, np.take_along_axis(lp, order, -1)


def token_log_probs_backward(x, ids, dlogp, dentropy, temperature=1.0):
    lp, m, _ = log_p(x, temperature)
    rows, vocab = lp.shape
    p = np.exp(lp)
    finite = np.where(p == 0, 0.0, lp)
    entropy = -(p * finite).sum(-1, keepdims=True)
    named = (ids >= 0) & (ids < vocab)
    a = np.zeros(rows) if dlogp is None else np.where(named, dlogp, 0.0)
    b = np.zeros(rows) if dentropy is None else np.asarray(dentropy, np.float64)
    hot = np.zeros_like(p)
    hot[np.arange(rows)[named], np.asarray(ids)[named]] = 1
    d = a[:, None] * (hot - p) - b[:, None] * p * (finite + entropy)
    return np.where((m == -np.inf)[:, None] | ((a == 0) & (b == 0))[:, None], 0.0, d / temperature)


def distill(x, teacher_ids, teacher, weight=None, temperature=1.0):
    """(loss, dlogits)."""
    rows, vocab = np.shape(x)
    lp, _, _ = log_p(x, temperature)
    loss, d = np.zeros(rows), np.zeros((rows, vocab))
    w = np.ones(rows) if weight is None else np.asarray(weight, np.float64)
    for r in range(rows):
        named = (teacher_ids[r] >= 0) & (teacher_ids[r] < vocab) & (teacher[r] > -np.inf)
        if not named.any():
            continue
        ids, u = np.asarray(teacher_ids[r])[named], np.asarray(teacher[r], np.float64)[named] / temperature
        u = u - u.max()
        log_t = u - np.log(np.exp(u).sum())
        t = np.exp(log_t)
        with np.errstate(invalid="ignore"):
            loss[r] = temperature ** 2 * np.where(t > 0, t * (log_t - lp[r][ids]), 0.0).sum()
        if w[r] != 0:
            d[r] = np.exp(lp[r])
            np.subtract.at(d[r], ids, t)
            d[r] *= w[r] * temperature
    return loss, d
