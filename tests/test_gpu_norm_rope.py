"""bc_norm_rope_split, its gradient and bc_norm_rope_decode_step against their fp64 oracle (oracle/norm_rope_oracle.py)."""
import math

import numpy as np
import pytest
import torch

from oracle.norm_rope_oracle import grad, heads, norm, norm_rope_split
from paper_2510_13797_b200 import binding as B
from tests.harness import Pair, f64, randn_bf16

pytestmark = pytest.mark.gpu
DEV = "cuda"
EPS = 1e-6


def _inputs(seed, n, Hq, Hkv, D, pad, far, weights=True):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    width = (Hq + 2 * Hkv) * D
    qkv = (randn_bf16(g, (n, width + pad), DEV, scale=2.0))[:, :width]
    pos = torch.randint(0, far, (n,), generator=g, device=DEV, dtype=torch.int32)
    pos[0] = 0
    wq, wk = [(1 + 0.3 * torch.randn(D, generator=g, device=DEV)).to(torch.bfloat16) if weights else None for _ in range(2)]
    return g, qkv, pos, wq, wk


def _w(w, D):
    return np.ones(D) if w is None else f64(w)


def _assert_forward(gpu, ref, y, what):
    """One rounding to bf16 (2^-8 of the value), and fp32 arithmetic ahead of it: a norm and a rotation are a dozen
    operations of 2^-24 and an angle off by 2^-23 turns, all relative to the pair (y[j], y[j + D/2]) that is turned: 1e-6 times 2."""
    half = y.shape[-1] // 2
    mag = np.tile(np.abs(y[..., :half]) + np.abs(y[..., half:]), 2)
    err = np.abs(f64(gpu) - ref) - (2.0 ** -8 * np.abs(ref) + 2e-6 * mag)
    assert err.max() <= 0, f"{what}: {err.max():.3e} over the bound"


SHAPES = [(12, 2, 128, 64, 0, 40000, True), (32, 8, 128, 77, 0, 131072, True), (4, 4, 64, 1, 0, 10, False), (14, 1, 64, 1031, 24, 9000, True),
          (1, 1, 128, 5, 8, 1 << 20, True), (7, 7, 128, 300, 64, 300, False)]


@pytest.mark.parametrize("Hq,Hkv,D,n,pad,far,weights", SHAPES)
def test_forward_matches_oracle(Hq, Hkv, D, n, pad, far, weights):
    _, qkv, pos, wq, wk = _inputs(3, n, Hq, Hkv, D, pad, far, weights)
    q, k, v = B.bc_norm_rope_split(qkv, pos, 1e6, wq, wk, EPS, Hq, Hkv)
    rq, rk, rv = norm_rope_split(f64(qkv), f64(pos), Hq, Hkv, D, 1e6, _w(wq, D), _w(wk, D), EPS)
    xq, xk, _ = heads(f64(qkv), Hq, Hkv, D)
    _assert_forward(q, rq, norm(xq, _w(wq, D), EPS), "q")
    _assert_forward(k, rk, norm(xk, _w(wk, D), EPS), "k")
    assert np.array_equal(f64(v), rv)


@pytest.mark.parametrize("Hq,Hkv,D,n,pad,far,weights", SHAPES)
def test_gradient_matches_formula(Hq, Hkv, D, n, pad, far, weights):
    g, qkv, pos, wq, wk = _inputs(4, n, Hq, Hkv, D, pad, far, weights)
    dq, dk, dv = [randn_bf16(g, (n, h, D), DEV) for h in (Hq, Hkv, Hkv)]
    dqkv, dwq, dwk = B.bc_norm_rope_split_backward(qkv, pos, 1e6, wq, wk, EPS, dq, dk, dv)
    xq, xk, _ = heads(f64(qkv), Hq, Hkv, D)
    out = f64(dqkv).reshape(n, Hq + 2 * Hkv, D)
    for x, w, go, got, gw, what in ((xq, wq, dq, out[:, :Hq], dwq, "q"), (xk, wk, dk, out[:, Hq:Hq + Hkv], dwk, "k")):
        dx, dw, mag, dw_mag = grad(x, _w(w, D), EPS, f64(pos), 1e6, f64(go))
        # the rotation mixes pairs of g (an angle off by 2^-23 turns), the mean adds D terms in fp32: 2e-6 of the largest term
        # of the head on top of the rounding to bf16
        bound = 2.0 ** -8 * np.abs(dx) + 2e-6 * mag.max(axis=-1, keepdims=True) * 4
        assert (np.abs(got - dx) - bound).max() <= 0, (what, (np.abs(got - dx) - bound).max())
        # at most about a hundred additions in a row (terms of a lane, lanes, warps, blocks), 2^-24 each, and the terms' own dozen;
        # the rotation again mixes coordinates: relative to the largest column
        assert np.all(np.abs(f64(gw) - dw) <= 1e-5 * dw_mag.max()), what
    assert np.array_equal(out[:, Hq + Hkv:], f64(dv))
    again = B.bc_norm_rope_split_backward(qkv, pos, 1e6, wq, wk, EPS, dq, dk, dv)
    assert all(torch.equal(a, b) for a, b in zip(again, (dqkv, dwq, dwk)))          # additions in a fixed order
    only = B.bc_norm_rope_split_backward(qkv, pos, 1e6, wq, wk, EPS, dq, dk, dv, weight_grads=False)
    assert torch.equal(only[0], dqkv) and only[1] is None


def test_gradient_along_a_direction_against_differences_of_the_oracle():
    """The gradient's inner product with a direction, against the change of the (fp64) loss along it."""
    n, Hq, Hkv, D = 40, 4, 2, 64
    g, qkv, pos, wq, wk = _inputs(5, n, Hq, Hkv, D, 0, 5000)
    dq, dk, dv = [randn_bf16(g, (n, h, D), DEV) for h in (Hq, Hkv, Hkv)]
    dqkv, dwq, dwk = B.bc_norm_rope_split_backward(qkv, pos, 1e4, wq, wk, EPS, dq, dk, dv)
    rng = np.random.RandomState(1)
    ux, uq, uk = rng.randn(*qkv.shape), rng.randn(D), rng.randn(D)

    def loss(t):
        q, k, v = norm_rope_split(f64(qkv) + t * ux, f64(pos), Hq, Hkv, D, 1e4, f64(wq) + t * uq, f64(wk) + t * uk, EPS)
        return (q * f64(dq)).sum() + (k * f64(dk)).sum() + (v * f64(dv)).sum()

    diff = (loss(1e-5) - loss(-1e-5)) / 2e-5
    terms = np.concatenate([(f64(dqkv) * ux).ravel(), f64(dwq) * uq, f64(dwk) * uk])
    # every term of the inner product is off by at most its rounding to bf16, 2^-8, with independent signs: 6 of their standard deviations
    assert abs(terms.sum() - diff) <= 6 * 2.0 ** -8 * math.sqrt((terms ** 2).sum())


def test_special_values_stay_in_their_head():
    Hq, Hkv, D, n = 4, 2, 128, 9
    _, qkv, pos, wq, wk = _inputs(6, n, Hq, Hkv, D, 0, 100)
    clean = B.bc_norm_rope_split(qkv, pos, 1e4, wq, wk, EPS, Hq, Hkv)
    bad = qkv.clone()
    bad[2, 5], bad[3, D + 7] = float("nan"), float("inf")
    bad[4, :D] = 0
    q, k, v = B.bc_norm_rope_split(bad, pos, 1e4, wq, wk, EPS, Hq, Hkv)
    assert bool(q[2, 0].isnan().all()) and bool(q[3, 1].isnan().any()) and float(q[4, 0].abs().max()) == 0.0
    keep = torch.ones((n, Hq), dtype=torch.bool, device=DEV)
    keep[2, 0] = keep[3, 1] = keep[4, 0] = False
    assert torch.equal(q[keep], clean[0][keep]) and torch.equal(k, clean[1]) and torch.equal(v, clean[2])


def test_given_outputs_streams_and_capture():
    Hq, Hkv, D, n = 12, 2, 128, 130
    _, qkv, pos, wq, wk = _inputs(7, n, Hq, Hkv, D, 8, 1000)
    want = B.bc_norm_rope_split(qkv, pos, 1e4, wq, wk, EPS, Hq, Hkv)
    q, k, v = [torch.full((n + 2, h, D), 7.0, dtype=torch.bfloat16, device=DEV) for h in (Hq, Hkv, Hkv)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    B.bc_norm_rope_split(qkv, pos, 1e4, wq, wk, EPS, Hq, Hkv, q[:n], k[:n], v[:n], stream=s)
    s.synchronize()
    assert all(torch.equal(a[:n], b) and float(a[n:].min()) == 7.0 for a, b in zip((q, k, v), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="thread_local"):
        B.bc_norm_rope_split(qkv, pos, 1e4, wq, wk, EPS, Hq, Hkv, q[:n], k[:n], v[:n])
        gd = B.bc_norm_rope_split_backward(qkv, pos, 1e4, wq, wk, EPS, q[:n], k[:n], v[:n])
    for t in range(2):
        qkv.mul_(-1) if t else q.zero_()
        graph.replay()
        want = B.bc_norm_rope_split(qkv, pos, 1e4, wq, wk, EPS, Hq, Hkv)
        assert all(torch.equal(a[:n], b) for a, b in zip((q, k, v), want))
        assert all(torch.equal(a, b) for a, b in zip(gd, B.bc_norm_rope_split_backward(qkv, pos, 1e4, wq, wk, EPS, q[:n], k[:n], v[:n])))


def test_binding_refuses_wrong_tensors():
    _, qkv, pos, wq, wk = _inputs(8, 4, 4, 2, 64, 0, 10)
    for bad in (dict(positions=pos.long()), dict(q_weight=wq.float()), dict(k_weight=wk[:32]), dict(qkv=qkv.float()), dict(qkv=qkv[:, :-8]),
                dict(positions=pos[:3]), dict(qkv=qkv.t()), dict(positions=pos.cpu())):
        args = dict(qkv=qkv, positions=pos, theta=1e4, q_weight=wq, k_weight=wk, eps=EPS, q_heads=4, kv_heads=2)
        args.update(bad)
        with pytest.raises(B.BreadcrumbsError) as e:
            B.bc_norm_rope_split(**args)
        assert e.value.status in (B.BC_ERR_INVALID_ARG, B.BC_ERR_UNSUPPORTED)


@pytest.mark.parametrize("L,Hkv,G,D", [(2, 2, 6, 128), (1, 1, 4, 64)])
def test_decode_step_is_the_two_calls(L, Hkv, G, D):
    Hq, n, scale = Hkv * G, 3, 1.0 / math.sqrt(D)
    a, b = [Pair(L, Hkv, Hq, D, 16, max_seqs=4, num_pages=200, max_pages_per_seq=50) for _ in range(2)]
    g, _, _, wq, wk = _inputs(9, 1, Hq, Hkv, D, 0, 10)
    plens, slots = [300, 0, 41], [0, 2, 3]
    for p in (a, b):
        p.open(slots, plens)
    for l in range(L):
        k, v = [randn_bf16(g, (sum(plens), Hkv, D), DEV) for _ in range(2)]
        for p in (a, b):
            p.prefill(l, slots, plens, k, v)
    sl = torch.tensor(slots, dtype=torch.int32, device=DEV)
    for t in range(3):
        pos = torch.tensor([x + t for x in plens], dtype=torch.int32, device=DEV)
        for l in range(L):
            qkv = randn_bf16(g, (n, (Hq + 2 * Hkv) * D), DEV)
            o1, o2 = a.gpu.new_out(n), b.gpu.new_out(n)
            a.gpu.bc_norm_rope_decode_step(l, sl, qkv, pos, 1e6, wq, wk, EPS, o1, scale)
            q, k, v = B.bc_norm_rope_split(qkv, pos, 1e6, wq, wk, EPS, Hq, Hkv)
            b.gpu.bc_decode_step(l, sl, q, k, v, o2, scale)
            assert torch.equal(o1, o2)
    assert a.gpu.bc_get_state(3) == b.gpu.bc_get_state(3)
    assert all(torch.equal(x, y) for x, y in zip(a.gpu.bc_export_seq(L - 1, 0, 303), b.gpu.bc_export_seq(L - 1, 0, 303)))
    with pytest.raises(B.BreadcrumbsError):                                          # nothing is appended twice per step
        a.gpu.bc_norm_rope_decode_step(1, sl, qkv, pos, 1e6, wq, wk, EPS, o1, scale)
    if L == 1:
        with pytest.raises(B.BreadcrumbsError):
            a.gpu.bc_norm_rope_decode_step(0, sl, qkv, pos, 1.0, wq, wk, EPS, o1, scale)
