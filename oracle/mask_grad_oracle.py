"""fp64 gradient of the mask form of one trajectory, from the definition: who sees what is written out as a matrix."""
import numpy as np


def visible(P, T, c):
    """Rows: T tokens, then the beacons.  Columns: prompt, beacons, tokens.  True where the row sees the column."""
    nb = T // c if c > 1 else 0
    see = np.zeros((T + nb, P + nb + T), dtype=bool)
    see[:, :P] = True
    for i in range(T):
        w = i // c if c > 1 else 0
        see[i, P:P + (w if c > 1 else 0)] = True
        see[i, P + nb + (w * c if c > 1 else 0):P + nb + i + 1] = True
    for m in range(nb):
        see[T + m, P:P + m + 1] = True
        see[T + m, P + nb + m * c:P + nb + (m + 1) * c] = True
    return see


def forward(see, q, k, v, scale):
    """One head: weights, outputs and the logarithms of the rows' sums.  q [rows, d], k, v [keys, d]."""
    z = np.where(see, scale * (q @ k.T), -np.inf)
    m = z.max(-1, keepdims=True)
    e = np.exp(z - m)
    return e / e.sum(-1, keepdims=True), (e / e.sum(-1, keepdims=True)) @ v, (m + np.log(e.sum(-1, keepdims=True)))[:, 0]


def grad(see, q, k, v, do, scale):
    """dq, dk, dv of one head, and for each of them the size of the terms that a calculation with weights and score gradients rounded to
    8 bits, and outputs rounded to 8 bits, may be off by 2^-8 of."""
    p, o, _ = forward(see, q, k, v, scale)
    dp = do @ v.T
    D = (do * o).sum(-1, keepdims=True)
    ds = p * (dp - D)
    off = np.abs(ds) + p * (np.abs(do) * np.abs(o)).sum(-1, keepdims=True)     # dS itself, and D from rounded outputs
    small = p * (np.abs(do) @ np.abs(v).T + np.abs(D))                         # what fp32 is relative to
    return ((scale * ds @ k, scale * off @ np.abs(k), scale * small @ np.abs(k)),
            (scale * ds.T @ q, scale * off.T @ np.abs(q), scale * small.T @ np.abs(q)),
            (p.T @ do, p.T @ np.abs(do), p.T @ np.abs(do)))
