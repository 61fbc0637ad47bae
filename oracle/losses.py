"""Base losses and top logits in float64 (NumPy), row by row from their definitions.

    cross entropy  l = -log q_y
    distillation   l = sum_k p_k (log p_k - log q_{i_k})
    gradient       scale w / T (P q - sum_k p_k e_{i_k}),  q = softmax(x / T)

label_members() and teacher_members() give every row's members; losses() the losses and the logits'
gradient for them; head() the same through an LM head.
"""
import numpy as np


def _lse(a):
    """log sum exp over the last axis (-inf where nothing is above it)."""
    top = np.max(a, axis=-1, keepdims=True)
    ref = np.where(np.isneginf(top), 0.0, top)
    with np.errstate(divide="ignore"):
        return (ref + np.log(np.sum(np.exp(a - ref), axis=-1, keepdims=True)))[..., 0]


def label_members(labels):
    """(idx [R, 1], p [R, 1], sum p log p [R]) of labels."""
    idx = np.asarray(labels, dtype=np.int64)[:, None]
    return idx, (idx >= 0).astype(np.float64), np.zeros(len(idx))


def teacher_members(idx, logits, lse=None, temp=1.0):
    """The same of a teacher's top logits."""
    idx = np.asarray(idx, dtype=np.int64)
    a = np.asarray(logits, dtype=np.float64) / temp
    a = np.where(idx < 0, -np.inf, a)
    z = _lse(a) if lse is None else np.asarray(lse, dtype=np.float64)
    z = np.where(np.isneginf(z), 0.0, z)
    logp = a - z[:, None]
    p = np.exp(logp)
    return idx, p, np.sum(np.where(p > 0, p * np.where(p > 0, logp, 0.0), 0.0), axis=1)


def losses(x, idx, p, plogp, weight=None, temp=1.0, scale=1.0):
    """dict(loss, lse, total, grad, q, live) of logits x [R, V] and members."""
    x = np.asarray(x, dtype=np.float64)
    R, V = x.shape
    w = np.ones(R) if weight is None else np.asarray(weight, dtype=np.float64)
    play = (np.sum(p, axis=1) != 0) & (w != 0)
    loss, lse, q, g = np.zeros(R), np.zeros(R), np.zeros((R, V)), np.zeros((R, V))
    for r in np.flatnonzero(play):
        a = x[r] / temp
        top = np.max(a)
        if np.isneginf(top):
            lse[r] = top
            continue
        # (against the maximum: log sum exp itself rounds at the logits' size)
        e = np.exp(a - top)
        tail = np.log(np.sum(e))
        lse[r], q[r] = top + tail, e / np.sum(e)
        on = p[r] > 0
        loss[r] = plogp[r] - np.sum(p[r][on] * (a[idx[r][on]] - top - tail))
        g[r] = np.sum(p[r]) * q[r]
        np.subtract.at(g[r], idx[r][on], p[r][on])
        g[r] *= scale * w[r] / temp
    return dict(loss=loss, lse=lse, total=scale * np.sum(np.where(loss != 0, w * loss, 0.0)), grad=g, q=q,
                live=play & ~np.isneginf(lse))


def head(h, w, members, weight=None, temp=1.0, scale=1.0):
    """losses() of x = h w^T, with grad_hidden and grad_weight (rows out of play
    may hold anything)."""
    h, w = np.asarray(h, dtype=np.float64), np.asarray(w, dtype=np.float64)
    idx, p, plogp = members
    play = np.sum(p, axis=1) != 0
    if weight is not None:
        play &= np.asarray(weight) != 0
    h = np.where(play[:, None], h, 0.0)
    out = losses(h @ w.T, idx, p, plogp, weight, temp, scale)
    out["grad_hidden"] = out["grad"] @ w
    out["grad_weight"] = out["grad"].T @ h
    return out


def top(y, k, d2t=None, temp=1.0):
    """(idx, logits, lse) of the k largest logits above -inf."""
    y = np.asarray(y, dtype=np.float64)
    cols = y if d2t is None else y[:, np.asarray(d2t)]
    R, n = cols.shape
    idx, val = np.full((R, k), -1, dtype=np.int64), np.full((R, k), -np.inf)
    for r in range(R):
        order = np.lexsort((np.arange(n), -cols[r]))
        order = order[cols[r][order] > -np.inf][:k]
        idx[r, :len(order)] = order
        val[r, :len(order)] = cols[r][order]
    return idx, val, _lse(y / temp)
