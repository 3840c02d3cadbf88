"""Slow fp64 reference of the one-head losses: cross entropy with labels and distillation from a teacher's top logits.

Test infrastructure only.  Heads are [V, H] here.  Both functions return loss, per_token_loss (0 for tokens that do not
count), grad_h, grad_W and dz = dL/dz without the common factor scale / (n tau), with which rounding bounds are formed.
"""
from __future__ import annotations

import numpy as np

RENORM, REST, DROP = 0, 1, 2


def log_softmax(z):
    z = z - z.max(axis=1, keepdims=True)
    return z - np.log(np.exp(z).sum(axis=1, keepdims=True))


def _finish(h, W, keep, rows, dz, factor, tau):
    n = int(keep.sum())
    rows = np.where(keep, rows * factor, 0.0)
    dz = np.where(keep[:, None], dz, 0.0)
    s = factor / (n * tau) if n else 0.0
    return dict(loss=rows.sum() / n if n else 0.0, per_token_loss=rows, dz=dz, s=s, n=n, grad_h=s * (dz @ W),
                grad_W=s * (dz.T @ h))


def cross_entropy(h, W, labels, mask=None, smoothing=0.0, z_loss=0.0, scale=1.0):
    h, W = np.asarray(h, np.float64), np.asarray(W, np.float64)
    labels = np.asarray(labels)
    T, V = h.shape[0], W.shape[0]
    keep = labels >= 0
    if mask is not None:
        keep = keep & (np.asarray(mask) != 0)
    h = np.where(keep[:, None], h, 0.0)
    z = h @ W.T
    lp = log_softmax(z)
    lse = (z - lp)[:, :1]
    q = np.full((T, V), smoothing / V)
    q[np.arange(T), np.maximum(labels, 0)] += 1 - smoothing
    rows = -(q * lp).sum(axis=1) + z_loss * lse[:, 0] ** 2
    p = np.exp(lp)
    dz = p * (1 + 2 * z_loss * lse) - q
    return _finish(h, W, keep, rows, dz, scale, 1.0)


def topk(top_logits, top_index, h, W, lse=None, mask=None, tau=1.0, tail=RENORM, scale=1.0, tau2=False):
    h, W = np.asarray(h, np.float64), np.asarray(W, np.float64)
    ids, a = np.asarray(top_index), np.asarray(top_logits, np.float64) / tau
    T, V = h.shape[0], W.shape[0]
    there = (ids >= 0) & (a > -np.inf)
    keep = there.any(axis=1)
    if mask is not None:
        keep = keep & (np.asarray(mask) != 0)
    h = np.where(keep[:, None], h, 0.0)
    lp = log_softmax(h @ W.T / tau)
    p = np.exp(lp)
    rows, dz = np.zeros(T), np.zeros((T, V))
    for t in range(T):
        if not keep[t]:
            continue
        at, x = ids[t][there[t]], a[t][there[t]]
        norm = x.max() + np.log(np.exp(x - x.max()).sum()) if tail == RENORM else float(lse[t])
        q = np.zeros(V)
        np.add.at(q, at, np.exp(x - norm))
        on = np.zeros(V, bool)
        on[at] = True
        pos = q > 0
        rows[t] = (q[pos] * (np.log(q[pos]) - lp[t][pos])).sum()
        dz[t] = q.sum() * p[t] - q
        if tail == REST:
            r = max(0.0, 1 - q.sum())
            if r > 0:
                out = p[t][~on].sum()
                rows[t] += r * (np.log(r) - np.log(out))
                dz[t] += r * (p[t] - np.where(on, 0.0, p[t] / out))
    return _finish(h, W, keep, rows, dz, scale * (tau * tau if tau2 else 1.0), tau)
