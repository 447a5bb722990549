"""CPU fp64 oracle of log probabilities of given tokens, entropies, the best
alternatives, and their gradients.

TEST INFRASTRUCTURE ONLY; shares no code with the CUDA path.  Written from the
definitions:

    l = logit_scale * z,  lse = log sum exp l,  q = exp(l - lse)
    logprob = l_y - lse,  entropy = - sum_j q_j log q_j
    dz = logit_scale * (r (1[j = y] - q_j) - h q_j (log q_j + entropy))

Pinned by closed forms and by differences in tests/test_logprob_oracle_pins.py.
"""

from __future__ import annotations

import numpy as np


def logprob_rows(z, targets, logit_scale=1.0):
    """(logprob, entropy, lse, log_q, counts) of rows of raw logits; ``targets`` None:
    every row counts and logprob is 0.  A row of -inf alone: lse and logprob -inf,
    entropy 0."""
    z = np.asarray(z, np.float64) * logit_scale
    T, V = z.shape
    counts = np.ones(T, bool) if targets is None else (np.asarray(targets) >= 0) & (np.asarray(targets) < V)
    logprob, entropy, lse, log_q = np.zeros(T), np.zeros(T), np.zeros(T), np.zeros((T, V))
    for t in np.flatnonzero(counts):
        top = z[t].max()
        lse[t] = top if top == -np.inf else top + np.log(np.exp(z[t] - top).sum())
        log_q[t] = -np.inf if top == -np.inf else z[t] - lse[t]
        some = log_q[t] > -np.inf
        entropy[t] = -(np.exp(log_q[t][some]) * log_q[t][some]).sum()
        if targets is not None:
            logprob[t] = log_q[t][targets[t]]
    return logprob, entropy, lse, log_q, counts


def logprob_grad(log_q, entropy, counts, targets, r=None, h=None, logit_scale=1.0):
    """Gradient of the raw logits; 0 for rows that do not count or hold -inf alone."""
    T, V = log_q.shape
    d = np.zeros((T, V))
    for t in np.flatnonzero(counts):
        some = log_q[t] > -np.inf
        if not some.any():
            continue
        q, lq = np.exp(log_q[t]), np.where(some, log_q[t], 0.0)
        if r is not None:
            d[t] -= r[t] * q
            d[t, targets[t]] += r[t]
        if h is not None:
            d[t] -= h[t] * q * (lq + entropy[t])
    return d * logit_scale


def best(z, top):
    """Columns of the ``top`` largest of every row, equal ones by rising column; a NaN
    counts as -inf."""
    z = np.where(np.isnan(z), -np.inf, np.asarray(z, np.float64))
    return np.argsort(-z, axis=1, kind="stable")[:, :top]
