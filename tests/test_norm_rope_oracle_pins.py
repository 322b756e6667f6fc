"""The norm-and-rotation oracle by hand and by differences, and the argument checks of the library's calls (no kernel runs)."""
import ctypes as C

import numpy as np

from oracle.norm_rope_oracle import grad, norm, norm_rope_split
from paper_2510_13797_b200 import binding as B


def test_norm_by_hand_and_position_zero():
    x = np.array([[3.0, 4.0, 0.0, 0.0]])                         # mean square 25 / 4
    assert np.allclose(norm(x, np.ones(4), 0.0), [[1.2, 1.6, 0, 0]])
    assert np.allclose(norm(x, [1, 2, 3, 4], 0.0), [[1.2, 3.2, 0, 0]])
    qkv = np.arange(1.0, 13.0).reshape(1, 12)
    q, k, v = norm_rope_split(qkv, [0], 1, 1, 4, 10.0, np.ones(4), np.ones(4), 1e-6)
    assert np.allclose(q[0, 0], norm(qkv[0, :4], np.ones(4), 1e-6)) and np.allclose(v[0, 0], [9, 10, 11, 12])
    q1, _, _ = norm_rope_split(qkv, [5], 1, 1, 4, 10.0, np.ones(4), np.ones(4), 1e-6)
    assert np.isclose((q1 ** 2).sum(), (q ** 2).sum()) and not np.allclose(q1, q)


def test_gradient_against_differences():
    rng = np.random.RandomState(0)
    n, h, d, eps, theta = 3, 2, 8, 1e-5, 100.0
    x, w, g, pos = rng.randn(n, h, d), rng.randn(d), rng.randn(n, h, d), np.array([0, 7, 1000])
    loss = lambda x, w: (norm_rope_split(np.concatenate([x, x, x], 1).reshape(n, -1), pos, h, h, d, theta, w, w, eps)[0] * g).sum()
    dx, dw, _, _ = grad(x, w, eps, pos, theta, g)
    t = 1e-6
    for at in [(0, 0, 0), (1, 1, 3), (2, 0, 7), (2, 1, 4)]:
        e = np.zeros_like(x); e[at] = t
        assert np.isclose((loss(x + e, w) - loss(x - e, w)) / (2 * t), dx[at], rtol=1e-6, atol=1e-8)
    for j in range(d):
        e = np.zeros(d); e[j] = t
        assert np.isclose((loss(x, w + e) - loss(x, w - e)) / (2 * t), dw[j], rtol=1e-6, atol=1e-8)


def test_calls_refuse_bad_arguments():
    lib, p = B.lib(), 1 << 20                                     # never dereferenced: refused on the host
    ok = [4, 12, 2, 128, p, 2048, p, 1e4, None, None, 1e-6, p, p, p, None]
    bad = [(0, 0), (1, 0), (2, 0), (4, None), (4, p + 2), (5, 2047), (5, 2040), (6, None), (7, 1.0), (8, p + 8), (10, -1.0), (11, None), (12, p + 4),
           (13, None)]
    for at, value in bad:
        args = list(ok)
        args[at] = value
        assert lib.bc_norm_rope_split(*args) == B.BC_ERR_INVALID_ARG, (at, value)
    assert lib.bc_norm_rope_split(*[96 if i == 3 else a for i, a in enumerate(ok)]) == B.BC_ERR_UNSUPPORTED
    size = C.c_size_t()
    assert lib.bc_norm_rope_query_bytes(128, C.byref(size)) == B.BC_OK and size.value > 0
    assert lib.bc_norm_rope_query_bytes(80, C.byref(size)) == B.BC_ERR_UNSUPPORTED and lib.bc_norm_rope_query_bytes(64, None) == B.BC_ERR_INVALID_ARG
    lib.bc_norm_rope_query_bytes(128, C.byref(size))
    ok = [4, 12, 2, 128, p, 2048, p, 1e4, None, None, 1e-6, p, p, p, p, p, p, p, size.value, None]
    for at, value in [(0, -1), (4, None), (11, None), (12, p + 8), (13, None), (14, None), (15, p + 2), (17, None), (18, size.value - 1), (5, 100)]:
        args = list(ok)
        args[at] = value
        assert lib.bc_norm_rope_split_backward(*args) == B.BC_ERR_INVALID_ARG, (at, value)


def test_cache_calls_refuse_a_null_cache():
    lib, p = B.lib(), 1 << 20
    assert lib.bc_chunk_attn(None, 0, p, p, p, 1, 1, p, p, 1.0, None) == B.BC_ERR_INVALID_ARG
    assert lib.bc_prefill_chunk(None, 0, p, p, p, 1, 1, p, p, p, p, 1.0, None) == B.BC_ERR_INVALID_ARG
    assert lib.bc_norm_rope_decode_step(None, 0, p, 1, p, p, 1e4, None, None, 1e-6, p, 1.0, None) == B.BC_ERR_INVALID_ARG
