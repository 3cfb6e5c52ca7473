"""Log probabilities of tokens in plain numpy, 64 bits.  Test infrastructure only."""
from __future__ import annotations

import numpy as np


def token_logprobs(logits, tokens, scale=1.0, n_top=0):
    """logits [R, V]; tokens int [R, n].  Returns (logp [R, n], entropy [R], top_ids [R, n_top], top_logp [R, n_top]), row after row."""
    x = np.asarray(logits, np.float64)
    R, V = x.shape
    tokens = np.asarray(tokens).reshape(R, -1)
    logp, entropy = np.empty(tokens.shape), np.empty(R)
    ids, top = np.full((R, n_top), -1), np.full((R, n_top), -np.inf)
    for i in range(R):
        bad = np.isnan(x[i]).any() or (x[i] == np.inf).any()
        some = np.flatnonzero(x[i] > -np.inf)
        if bad:
            lp, entropy[i], top[i] = np.full(V, np.nan), np.nan, np.nan
        elif not len(some):
            lp, entropy[i] = np.full(V, -np.inf), 0.0
        else:
            z = scale * x[i, some]
            z = z - z.max()
            w = np.exp(z)
            lp = np.full(V, -np.inf)
            lp[some] = z - np.log(w.sum())
            entropy[i] = -(np.exp(lp[some]) * lp[some]).sum()
            order = some[np.argsort(-x[i, some], kind="stable")][:n_top]
            ids[i, :len(order)], top[i, :len(order)] = order, lp[order]
        for j, t in enumerate(tokens[i]):
            logp[i, j] = 0.0 if t < 0 else np.nan if t >= V else lp[t]
    return logp, entropy, ids, top


def token_logprobs_limits(logits, scale=1.0):
    """How far the kernel's sums may take a row from 64 bits: (a [R], b [R]), with |error of a log probability| <= a + 2^-21 |it| and
    |error of the entropy| <= b.

    In single precision, u = 2^-24.  An exponent d = k x + down is rounded once (u |d|), its factor k = scale log2(e) twice (2 u of
    |x - max| k, as what is common to a row cancels), exp2 and log2 are right to 2 u; a lane adds V / 256 weights at most, the row
    16 sums more, each of which rounds.  So with A = sum p |z - max| + 8 (8: what a wave's `down` may be short of its maximum by, in
    exponents of 2) the weights' sum is off by ((V / 256 + 20) + 4 A) u of itself, its logarithm by as much and 2 u of itself, and the sum of weights
    times exponents by ((V / 256 + 24) + 4) u A and 4 u times the sum of p (z - max)^2."""
    x = np.asarray(logits, np.float64)
    u, n = 2.0 ** -24, x.shape[1] / 256
    a, b = np.zeros(len(x)), np.zeros(len(x))
    for i, row in enumerate(x):
        some = row[row > -np.inf]
        if not len(some) or not np.isfinite(some).all():
            continue
        z = scale * some
        z = z - z.max()
        w = np.exp(z)
        p, ls = w / w.sum(), np.log(w.sum())
        A, B = (p * np.abs(z)).sum() + 8, (p * z * z).sum()
        a[i] = (n + 20 + 4 * A + 4 * (ls + 8)) * u
        b[i] = a[i] + ((n + 28) * A + 4 * B) * u
    return a, b
