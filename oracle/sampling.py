"""Sampling from (allowed) logits by given numbers, in fp64, row by row (an extension: Section 3.3 ranks).

Candidates of a row: tokens that are allowed and whose logit is not -inf, in the order (logit descending, token
ascending).  With w = e^((logit - max) / T): top-k keeps the first k of them; top-p of these the fewest, from the first
on, whose w reach p of the sum of their w; min-p of these those with w >= q, the first always.  A draw takes the first
kept token in ascending order at which the running sum of kept w exceeds u times the whole.  T <= 0 or NaN: the first
candidate.  A largest logit of +inf: those at +inf weigh 1, all others nothing."""
from __future__ import annotations

import numpy as np


def kept_tokens(logits, allow, T, k, p, q):
    """(tokens ascending, their weights) that the limits leave of one row; None without a candidate."""
    x = np.asarray(logits, dtype=np.float64)
    cand = np.flatnonzero((x > -np.inf) if allow is None else (np.asarray(allow, bool) & (x > -np.inf)))
    if cand.size == 0:
        return None
    order = cand[np.lexsort((cand, -x[cand]))]
    top = x[order[0]]
    if not T > 0:
        return order[:1], np.ones(1)
    if top == np.inf:
        order = order[x[order] == np.inf]
        w = np.ones(order.size)
    else:
        w = np.exp((x[order] - top) / T)
    n = order.size if k <= 0 else min(k, order.size)
    if p < 1:
        total, run, m = w[:n].sum(), 0.0, 0
        while m < n:
            run += w[m]
            m += 1
            if run >= p * total:
                break
        n_p = m
    else:
        n_p = n
    if q > 0:
        n_p = max(1, min(n_p, int(np.count_nonzero(w[:n] >= min(q, 1.0)))))
    kept, wk = order[:n_p], w[:n_p]
    by_token = np.argsort(kept)
    return kept[by_token], wk[by_token]


def sample_row(logits, allow, T, k, p, q, u):
    """(tokens [n], log q [n]) of the draws u of one row; tokens 0 and log q -inf without a candidate."""
    kept = kept_tokens(logits, allow, T, k, p, q)
    if kept is None:
        return np.zeros(len(u), np.int64), np.full(len(u), -np.inf)
    tokens, w = kept
    run = np.cumsum(w)
    at = np.minimum(np.searchsorted(run, np.asarray(u, np.float64) * run[-1], side="right"), len(tokens) - 1)
    return tokens[at], np.log(w[at] / run[-1])
