"""bc_norm_rope_split and its gradient where a warp has several rows and several passes per row, against the fp64 oracle
(oracle/norm_rope_oracle.py), and the weights' gradients over millions of rows."""
import numpy as np
import pytest
import torch

from oracle.norm_rope_oracle import grad, heads, norm, norm_rope_split
from paper_2510_13797_b200 import binding as B
from tests.harness import f64, randn_bf16
from tests.test_gpu_norm_rope import EPS, _assert_forward, _inputs, _w

pytestmark = pytest.mark.gpu
DEV = "cuda"

# More units than the 2368 warps of the grid, in one pass per unit and in several.
SHAPES = [(14, 1, 64, 5000, 8, 9000, True), (14, 1, 128, 2500, 0, 70000, True), (32, 8, 128, 2500, 0, 131072, False), (32, 8, 64, 5000, 24, 5000, True),
          (1, 1, 64, 12001, 0, 400, True)]


@pytest.mark.parametrize("Hq,Hkv,D,n,pad,far,weights", SHAPES)
def test_forward_of_several_units_and_passes_per_warp(Hq, Hkv, D, n, pad, far, weights):
    _, qkv, pos, wq, wk = _inputs(41, n, Hq, Hkv, D, pad, far, weights)
    q, k, v = B.bc_norm_rope_split(qkv, pos, 1e6, wq, wk, EPS, Hq, Hkv)
    rq, rk, rv = norm_rope_split(f64(qkv), f64(pos), Hq, Hkv, D, 1e6, _w(wq, D), _w(wk, D), EPS)
    xq, xk, _ = heads(f64(qkv), Hq, Hkv, D)
    _assert_forward(q, rq, norm(xq, _w(wq, D), EPS), "q")
    _assert_forward(k, rk, norm(xk, _w(wk, D), EPS), "k")
    assert np.array_equal(f64(v), rv)


@pytest.mark.parametrize("Hq,Hkv,D,n,pad,far,weights", SHAPES)
def test_gradient_of_several_units_and_passes_per_warp(Hq, Hkv, D, n, pad, far, weights):
    g, qkv, pos, wq, wk = _inputs(42, n, Hq, Hkv, D, pad, far, weights)
    dq, dk, dv = [randn_bf16(g, (n, h, D), DEV) for h in (Hq, Hkv, Hkv)]
    dqkv, dwq, dwk = B.bc_norm_rope_split_backward(qkv, pos, 1e6, wq, wk, EPS, dq, dk, dv)
    xq, xk, _ = heads(f64(qkv), Hq, Hkv, D)
    out = f64(dqkv).reshape(n, Hq + 2 * Hkv, D)
    for x, w, go, got, gw, what in ((xq, wq, dq, out[:, :Hq], dwq, "q"), (xk, wk, dk, out[:, Hq:Hq + Hkv], dwk, "k")):
        dx, dw, mag, dw_mag = grad(x, _w(w, D), EPS, f64(pos), 1e6, f64(go))
        # the rotation mixes pairs of g (an angle off by 2^-23 turns), the mean adds D terms in fp32: 2e-6 of the largest term
        # of the head, times 4, on top of the rounding to bf16
        bound = 2.0 ** -8 * np.abs(dx) + 8e-6 * mag.max(axis=-1, keepdims=True)
        assert (np.abs(got - dx) - bound).max() <= 0, (what, (np.abs(got - dx) - bound).max())
        # a lane adds at most 128 terms up before they go to the warp's sum; with the few dozen additions of warps and blocks and the
        # dozen operations of a term 200 times 2^-24 is 1.2e-5, relative to the largest column since the rotation mixes columns
        assert np.all(np.abs(f64(gw) - dw) <= 1.2e-5 * dw_mag.max()), what
    assert np.array_equal(out[:, Hq + Hkv:], f64(dv))
    again = B.bc_norm_rope_split_backward(qkv, pos, 1e6, wq, wk, EPS, dq, dk, dv)
    assert all(torch.equal(a, b) for a, b in zip(again, (dqkv, dwq, dwk)))


@pytest.mark.parametrize("D", [64, 128])
def test_weight_gradients_over_millions_of_rows(D):
    """Equal terms, each a little more than a number that fp32 sums of a thousand of them can hold: a sum of 1700 in a row (a lane's terms
    here) would lose 388 times 2^-24.  Allowed: 128 additions per lane, 14 of these sums, 3 between lanes, 8 warps, 42 in the last
    kernel, and 8 roundings of the term itself: 203 times 2^-24."""
    n = 2368 * 1700
    qkv = torch.ones((n, 3 * D), dtype=torch.bfloat16, device=DEV)
    g = torch.full((n, 1, D), 1.0078125, dtype=torch.bfloat16, device=DEV)
    # the term x r g is to be 1 + 0.49 * 2^-13
    eps = float(np.float32((1.0078125 / (1 + 0.49 * 2.0 ** -13)) ** 2 - 1))
    pos = torch.zeros(n, dtype=torch.int32, device=DEV)
    dqkv, dwq, dwk = B.bc_norm_rope_split_backward(qkv, pos, 1e4, None, None, eps, g, g, g)
    want = n * 1.0078125 / np.sqrt(1 + eps)
    for dw in (dwq, dwk):
        assert np.abs(f64(dw) / want - 1).max() <= 203 * 2.0 ** -24
    dx = 1.0078125 / np.sqrt(1 + eps) * (1 - 1 / (1 + eps))
    assert (dqkv[:, :2 * D].amin().item(), dqkv[:, :2 * D].amax().item()) == (pytest.approx(dx, rel=2.0 ** -8 + 1e-4),) * 2
