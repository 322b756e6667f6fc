"""The oracles of the training operators against differences and closed forms, and the library's refusals; no kernel runs here."""
import ctypes as C

import numpy as np
import pytest

from oracle import block_norm_oracle as BN
from oracle import logprobs_oracle as LP
from paper_2510_13797_b200 import binding as B


def test_logprobs_of_a_uniform_and_of_a_two_point_row():
    given, entropy, (m, ls), order, top = LP.logprobs(np.full(8, 3.0), 5, 3)
    assert np.isclose(given, -np.log(8)) and np.isclose(entropy, np.log(8)) and (m, list(order)) == (3.0, [0, 1, 2])
    assert np.allclose(top, -np.log(8)) and np.isclose(ls, np.log(8))
    given, entropy, _, order, top = LP.logprobs(np.array([-np.inf, np.nan, 0.0, np.log(3.0)]), 0, 4)
    assert given == -np.inf and list(order) == [3, 2, 0, 1] and np.allclose(top[:2], np.log([0.75, 0.25])) and (top[2:] == -np.inf).all()
    assert np.isclose(entropy, -(0.75 * np.log(0.75) + 0.25 * np.log(0.25)))
    assert LP.logprobs(np.array([np.inf, 1.0, np.inf]), 2, 1)[0] == pytest.approx(np.log(0.5))
    assert LP.logprobs(np.array([-np.inf, -np.inf]), 1, 1)[1] == 0 and not LP.grad(np.array([-np.inf, np.nan]), 0, 1.0, 1.0)[0].any()


def test_logprobs_gradient_against_differences():
    rng = np.random.RandomState(0)
    x, d, g, h = rng.randn(60) * 2, rng.randn(60), 0.7, -0.3
    loss = lambda t: (lambda r: g * r[0] + h * r[1])(LP.logprobs(x + t * d, 17, 1))
    e = 1e-5
    assert (LP.grad(x, 17, g, h)[0] @ d) == pytest.approx((loss(e) - loss(-e)) / (2 * e), rel=1e-7)
    assert (LP.grad(x, -100, g, h)[0] @ d) == pytest.approx(h * (LP.logprobs(x + e * d, 0, 1)[1] - LP.logprobs(x - e * d, 0, 1)[1]) / (2 * e), rel=1e-7)


@pytest.mark.parametrize("post", [True, False])
def test_block_norm_gradient_against_differences(post):
    rng = np.random.RandomState(1)
    n, hid, eps, scale = 3, 24, 1e-3, 0.6
    x, h, a, b = [rng.randn(n, hid) for _ in range(4)]
    gate, w1, w2 = rng.randn(hid), rng.randn(hid), rng.randn(hid)
    dirs = [rng.randn(*t.shape) for t in (x, h, gate, w1, w2)]

    def loss(t):
        xx, hh, gg, p, q = [v + t * d for v, d in zip((x, h, gate, w1, w2), dirs)]
        new = BN.stream(xx, hh, gg, post, p, scale, eps)
        return (a * new).sum() + (b * BN.unit(new, q, eps)).sum()
    dx, dh, dg, dp, dq = BN.grad(x, BN.stream(x, h, gate, post, w1, scale, eps), gate, post, w1, w2, scale, eps, a, b)
    want = (dx * dirs[0]).sum() + (dh * dirs[1]).sum() + (dg.sum(0) * dirs[2]).sum() + (dp.sum(0) * dirs[3]).sum() + (dq.sum(0) * dirs[4]).sum()
    assert want == pytest.approx((loss(1e-5) - loss(-1e-5)) / 2e-5, rel=1e-6)


P = C.c_void_p(1 << 20)          # an aligned address that no refused call touches
ODD = C.c_void_p((1 << 20) + 1)
LOGP = dict(logits=P, f32=0, stride=100, n=4, vocab=100, targets=P, top_k=5, logprob=P, entropy=P, stats=P, idx=P, top=P, stream=None)
LOGP_GRAD = dict(logits=P, f32=0, stride=100, n=4, vocab=100, targets=P, stats=P, entropy=P, dl=P, de=P, grad=P, gstride=100, stream=None)
NORM = dict(n=4, hidden=64, x=P, h=P, gate=P, gstride=0, post=1, pw=P, qw=P, scale=1.0, eps=1e-6, out=P, y=P, stream=None)
NORM_GRAD = dict(n=4, hidden=64, x=P, h=P, gate=P, gstride=0, post=1, pw=P, qw=P, scale=1.0, eps=1e-6, a=P, b=P, dx=P, dh=P, dg=P, dp=P, dq=P, ws=P,
                 size=1 << 40, stream=None)
INVALID, UNSUPPORTED = B.BC_ERR_INVALID_ARG, B.BC_ERR_UNSUPPORTED


@pytest.mark.parametrize("name,args,change,want", [
    ("bc_token_logprobs", LOGP, c, w) for c, w in [
        (dict(logits=None), INVALID), (dict(logits=ODD), INVALID), (dict(f32=1, logits=C.c_void_p((1 << 20) + 2)), INVALID), (dict(f32=2), INVALID),
        (dict(stride=99), INVALID), (dict(n=0), INVALID), (dict(vocab=0), INVALID), (dict(targets=None), INVALID), (dict(top_k=-1), INVALID),
        (dict(top_k=101), INVALID), (dict(idx=None), INVALID), (dict(top=None), INVALID), (dict(entropy=ODD), INVALID), (dict(targets=ODD), INVALID),
        (dict(vocab=300000, stride=300000), UNSUPPORTED), (dict(vocab=1000, stride=1000, top_k=257), UNSUPPORTED)]] + [
    ("bc_token_logprobs_backward", LOGP_GRAD, c, w) for c, w in [
        (dict(logits=None), INVALID), (dict(stats=None), INVALID), (dict(grad=None), INVALID), (dict(gstride=99), INVALID), (dict(targets=None), INVALID),
        (dict(entropy=None), INVALID), (dict(dl=None, de=None), INVALID), (dict(grad=ODD), INVALID), (dict(dl=ODD), INVALID), (dict(n=-3), INVALID),
        (dict(vocab=262145, stride=262145, gstride=262145), UNSUPPORTED)]] + [
    ("bc_block_norm", NORM, c, w) for c, w in [
        (dict(x=None), INVALID), (dict(h=None), INVALID), (dict(out=None), INVALID), (dict(n=0), INVALID), (dict(hidden=0), INVALID),
        (dict(gstride=32), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(y=ODD), INVALID),
        (dict(pw=ODD), INVALID), (dict(hidden=60), UNSUPPORTED), (dict(hidden=8200), UNSUPPORTED)]] + [
    ("bc_block_norm_backward", NORM_GRAD, c, w) for c, w in [
        (dict(a=None, b=None), INVALID), (dict(dx=None), INVALID), (dict(dh=None), INVALID), (dict(ws=None), INVALID), (dict(size=100), INVALID),
        (dict(gate=None), INVALID), (dict(post=0), INVALID), (dict(dp=ODD), INVALID), (dict(dx=ODD), INVALID), (dict(hidden=12), UNSUPPORTED)]])
def test_refusals_on_the_host(name, args, change, want):
    assert getattr(B.lib(), name)(*{**args, **change}.values()) == want


def test_workspace_sizes():
    size = C.c_size_t()
    for hidden in (8, 1536, 8192):
        assert B.lib().bc_block_norm_query_bytes(hidden, C.byref(size)) == 0 and size.value >= 12 * hidden
    assert B.lib().bc_block_norm_query_bytes(9000, C.byref(size)) == UNSUPPORTED and B.lib().bc_block_norm_query_bytes(64, None) == INVALID
