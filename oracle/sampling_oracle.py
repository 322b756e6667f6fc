"""Sampling of one token from a row of logits, fp64 (TEST INFRASTRUCTURE ONLY).

Algorithm 1 samples the next token from the model's distribution; temperature, top-k, top-p and min-p are the
usual restrictions of it.  The definition, for a row x with maximum m and e_j = exp((x_j - m) / T):
the top_k largest (ties: lowest index), of these the shortest prefix whose mass reaches top_p of theirs, of these the
elements with e_j >= min_p; the token is the first of them in index order at which the running mass exceeds
u times the whole.

Pinned by tests/test_sampling_oracle_pins.py.
"""
import numpy as np


def kept(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Indices of the elements that may be chosen, ascending, and their unnormalised weights.  temperature > 0."""
    x = np.asarray(x, dtype=np.float64)
    x = np.where(np.isnan(x), -np.inf, x) + 0.0
    m = x.max()
    with np.errstate(invalid="ignore", over="ignore"):
        e = np.where(x == m, 1.0, np.where(np.isneginf(x), 0.0, np.exp((x - m) / float(temperature))))
    order = np.lexsort((np.arange(x.size), -x))
    if 0 < top_k < x.size:
        order = order[:top_k]
    if top_p < 1:
        c = np.cumsum(e[order])
        order = order[:1 + int(np.sum(c[:-1] < top_p * c[-1]))]
    idx = np.sort(order)
    if min_p > 0:
        idx = idx[e[idx] >= min(min_p, 1.0)]
    return idx, e[idx]


def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    x = np.asarray(x, dtype=np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    if not temperature > 0 or x.max() == -np.inf:
        return int(np.argmax(x))
    idx, e = kept(x, temperature, top_k, top_p, min_p)
    u = min(max(float(u), 0.0), 1.0 - 2.0 ** -24) if u == u else 0.0
    c = np.cumsum(e)
    return int(idx[min(int(np.sum(c <= u * c[-1])), len(idx) - 1)])
