"""Attention of a chunk of queries over the first entries of a sequence, fp64 (TEST INFRASTRUCTURE ONLY).

Row r sees the first `first + r + 1` of the entries K, V (Section 2, ordinary softmax attention over what is
visible); zeros where that is none."""
import numpy as np


def chunk_attend(q, K, V, first, scale):
    """q [m, Hq, D]; K, V [entries, Hkv, D] -> (out [m, Hq, D], sum of weight * |V|, the size the rounding bounds refer to)."""
    m, hq, d = q.shape
    g = hq // K.shape[1] if K.shape[0] else 1
    out, mag = np.zeros((m, hq, d)), np.zeros((m, hq, d))
    for r in range(m):
        vis = min(max(first + r + 1, 0), K.shape[0])
        if vis == 0:
            continue
        for h in range(hq):
            s = K[:vis, h // g] @ q[r, h] * scale
            w = np.exp(s - s.max())
            w /= w.sum()
            out[r, h], mag[r, h] = w @ V[:vis, h // g], w @ np.abs(V[:vis, h // g])
    return out, mag
