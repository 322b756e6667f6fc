"""fp64 definition of bc_token_logprobs and its gradient, row by row, from the formulas."""
import numpy as np

FAR = 2.0 ** 126


def clean(x):
    """Logits as they count: NaN and -inf without mass (-inf), the others no further from 0 than 2^126."""
    x = np.where(np.isnan(x), -np.inf, x)
    return np.where(x <= -FAR, -np.inf, np.minimum(x, FAR))


def log_p(x):
    """(log p, maximum, ln s) of one row; maximum -inf where there is no distribution."""
    y = clean(x)
    m = y.max()
    if m == -np.inf:
        return np.full(y.shape, -np.inf), -np.inf, 0.0
    ls = np.log(np.exp(y - m).sum())
    return (y - m) - ls, m, ls


def logprobs(x, target, top_k):
    """logprob, entropy, stats, top indices, top log-probabilities of one row."""
    lp, m, ls = log_p(x)
    p = np.exp(lp)
    entropy = -np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0).sum()
    order = np.lexsort((np.arange(x.size), -np.where(np.isnan(x), -np.inf, x + 0.0)))[:top_k]
    given = lp[target] if 0 <= target < x.size else 0.0
    return given, entropy, (m, ls), order, lp[order]


def grad(x, target, g, h):
    """d loss / d x of one row and the size of the terms it is made of."""
    lp, m, _ = log_p(x)
    if m == -np.inf:
        return np.zeros(x.shape), np.zeros(x.shape)
    p = np.exp(lp)
    safe = np.where(p > 0, lp, 0.0)
    entropy = -(p * safe).sum()
    hot = np.zeros(x.shape)
    if 0 <= target < x.size:
        hot[target] = 1.0
    else:
        g = 0.0
    size = np.abs(g) * (hot + p) + np.abs(h) * p * (np.abs(safe) + entropy)
    return g * (hot - p) - h * p * (safe + entropy), size
