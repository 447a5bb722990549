"""CPU fp64 oracle of the losses at the LM head and their gradients.

TEST INFRASTRUCTURE ONLY; shares no code with the CUDA path.  Written from the
definitions:

    l = logit_scale * x w^T / temperature,  lse = log sum exp l,  q = exp(l - lse)
    cross entropy   loss = lse - l_target + z_loss lse^2
    distillation    loss = sum_k p_k (log p_k - (l_k - lse)),
                    p = softmax(z / temperature) over the entries, or
                    exp(z / temperature - teacher_lse)

``total = sum_t g_t loss_t`` with g = scale * weight (mean: over the sum of the
weights of the tokens that are not masked); dx and dw are its gradients.  Pinned
by closed forms, by differences and by hand in tests/test_head_oracle_pins.py.
"""

from __future__ import annotations

import numpy as np


def target_rows(targets, vocab):
    """Cross entropy as sparse distributions: (ids [T, 1], p [T, 1], usable [T, 1])."""
    ids = np.asarray(targets)[:, None]
    usable = (ids >= 0) & (ids < vocab)
    return np.where(usable, ids, 0), usable.astype(np.float64), usable


def teacher_rows(ids, z, vocab, temperature, teacher_lse=None):
    """A teacher's entries as sparse distributions."""
    ids, z = np.asarray(ids), np.asarray(z, np.float64) / temperature
    usable = (ids >= 0) & (ids < vocab) & ~(z == -np.inf)
    p = np.zeros_like(z)
    for t in range(ids.shape[0]):
        k = usable[t]
        if k.any():
            ref = np.log(np.exp(z[t, k] - z[t, k].max()).sum()) + z[t, k].max() if teacher_lse is None else teacher_lse[t]
            p[t, k] = np.exp(z[t, k] - ref)
    return np.where(usable, ids, 0), p, usable


def head_loss(x, w, rows, weight=None, mean=True, scale=1.0, logit_scale=1.0, temperature=1.0, z_loss=0.0, grads=True):
    """``rows``: what target_rows / teacher_rows give.  Returns a dict with loss,
    lse, total, dx, dw, the gradient ``g`` of the raw logits and ``bound_dx``,
    ``bound_dw``: the same products of absolute values, which rounding errors of
    the operands are measured against."""
    for a in (x, w):
        if np.asarray(a).dtype != np.float64:
            raise TypeError("oracle inputs must already be widened to float64")
    ids, p, usable = rows
    T, V = x.shape[0], w.shape[0]
    counts = usable.any(axis=1)
    wt = np.ones(T) if weight is None else np.asarray(weight, np.float64)
    norm = wt[counts].sum()
    g = np.where(counts, scale * wt, 0.0)
    if mean:
        g = g / norm if norm != 0 else np.zeros(T)
    loss, lse, G = np.zeros(T), np.zeros(T), np.zeros((T, V))
    a = logit_scale / temperature
    for t in np.flatnonzero(counts):
        l = a * (w @ x[t])
        top = l.max()
        lse[t] = top + np.log(np.exp(l - top).sum())
        log_q = l - lse[t]
        k = p[t] > 0
        loss[t] = (p[t, k] * (np.log(p[t, k]) - log_q[ids[t, k]])).sum() + z_loss * lse[t] ** 2
        d = (p[t].sum() + 2 * z_loss * lse[t]) * np.exp(log_q)
        np.add.at(d, ids[t], -p[t])
        G[t] = g[t] * a * d
    out = {"loss": loss, "lse": lse, "total": float((g * loss).sum()), "g": G, "counts": counts}
    if grads:
        xs = np.where(counts[:, None], x, 0.0)
        out.update(dx=G @ w, dw=G.T @ xs, bound_dx=np.abs(G) @ np.abs(w), bound_dw=np.abs(G).T @ np.abs(xs))
    return out
