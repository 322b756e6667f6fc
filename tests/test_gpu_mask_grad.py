"""bc_mask_attn_forward_lse and bc_mask_attn_backward against the fp64 definition (oracle/mask_grad_oracle.py)."""
import math

import numpy as np
import pytest
import torch

from oracle import mask_grad_oracle as O
from paper_2510_13797_b200 import binding as B
from tests.harness import f64, randn_bf16

pytestmark = pytest.mark.gpu
DEV = "cuda"
D = 128
NAMES = ("prompt_k", "prompt_v", "tok_q", "tok_k", "tok_v", "beacon_q", "beacon_k", "beacon_v")


def _case(seed, P, T, c, Hq, Hkv, spread=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    nb = [t // c if c > 1 else 0 for t in T]
    rows = dict(prompt=sum(P), tok=sum(T), beacon=sum(nb))
    x = {k: randn_bf16(g, (rows[k.split("_")[0]], Hq if k.endswith("q") else Hkv, D), DEV, scale=spread if k[-1] != "v" else 1.0) for k in NAMES}
    return x, [randn_bf16(g, (rows[k], Hq, D), DEV) for k in ("tok", "beacon")], nb


def _run(x, do, P, T, c, scale, **kw):
    ins = [x[k] for k in NAMES]
    out = B.bc_mask_attn_forward_lse(P, T, c, *ins, scale)
    return out, B.bc_mask_attn_backward(P, T, c, *ins, *out, *do, scale, **kw)


def _check(x, do, nb, P, T, c, Hq, Hkv, scale, out, grads, sequences=None):
    X, dO = {k: f64(v) for k, v in x.items()}, [f64(t) for t in do]
    got = dict(zip(NAMES, (f64(t) for t in grads)))
    lse = [f64(t) for t in out[2:]]
    G = Hq // Hkv
    for i in range(len(T)) if sequences is None else sequences:
        cut = lambda ln: slice(sum(ln[:i]), sum(ln[:i + 1]))
        cp, ct, cb = cut(P), cut(T), cut(nb)
        if T[i] == 0:                                     # no row sees the prompt
            assert not got["prompt_k"][cp].any() and not got["prompt_v"][cp].any()
            continue
        see = O.visible(P[i], T[i], c)
        for h in range(Hkv):
            k = np.concatenate([X["prompt_k"][cp, h], X["beacon_k"][cb, h], X["tok_k"][ct, h]])
            v = np.concatenate([X["prompt_v"][cp, h], X["beacon_v"][cb, h], X["tok_v"][ct, h]])
            sums = [0, 0]
            for hq in range(h * G, (h + 1) * G):
                q = np.concatenate([X["tok_q"][ct, hq], X["beacon_q"][cb, hq]])
                g = np.concatenate([dO[0][ct, hq], dO[1][cb, hq]])
                _, _, want = O.forward(see, q, k, v, scale)
                mine = np.concatenate([lse[0][ct, hq], lse[1][cb, hq]])
                # fp32: scores of 128 terms, weights to 2^-22, sums of some hundreds of additions
                assert np.all(np.abs(mine - want) <= 2e-5 * (1 + np.abs(want))), ("lse", np.abs(mine - want).max())
                (dq, off, small), dk, dv = O.grad(see, q, k, v, g, scale)
                mine = np.concatenate([got["tok_q"][ct, hq], got["beacon_q"][cb, hq]])
                _close("dq", mine, dq, off, small)
                sums = [tuple(a + b for a, b in zip(s, t)) if s else t for s, t in zip(sums, (dk, dv))]
            for what, (ref, off, small) in zip("kv", sums):
                mine = np.concatenate([got["prompt_" + what][cp, h], got["beacon_" + what][cb, h], got["tok_" + what][ct, h]])
                _close("d" + what, mine, ref, off, small)


def _close(what, got, ref, off, small):
    """Roundings to bf16 of the factor of the second product, of the outputs in D and of the result, half a step (2^-8) each; and fp32:
    scores and row sums to 2e-5 of the weights, products of 128 terms, accumulation over the rows."""
    err = np.abs(got - ref) - (2.0 ** -8 * (np.abs(ref) + off) + 1e-4 * small + 1e-30)
    assert err.max() <= 0, (what, err.max(), np.unravel_index(err.argmax(), err.shape))


CASES = [  # P, T, c, Hq, Hkv
    ([1], [1], 1, 1, 1), ([0], [1], 4, 2, 2), ([5], [3], 4, 4, 1), ([0], [64], 16, 4, 2), ([70], [333], 16, 12, 2), ([128], [128], 1, 8, 2),
    ([129], [257], 2, 4, 4), ([0], [700], 1, 2, 1), ([300, 0, 64], [65, 400, 1], 8, 14, 2), ([33, 500], [130, 129], 50, 16, 1), ([10, 20], [31, 5], 32, 6, 2),
    ([90], [520], 2, 10, 2), ([0, 7], [0, 40], 4, 4, 2), ([40, 9], [20, 0], 4, 4, 2), ([200], [260], 128, 3, 1), ([1], [200], 200, 5, 1), ([64], [2050], 2, 2, 2)]


@pytest.mark.parametrize("P,T,c,Hq,Hkv", CASES)
def test_gradient_matches_the_definition(P, T, c, Hq, Hkv):
    x, do, nb = _case(sum(P) + sum(T), P, T, c, Hq, Hkv)
    scale = 1 / math.sqrt(D)
    out, grads = _run(x, do, P, T, c, scale)
    plain = B.bc_mask_attn_forward(P, T, c, *[x[k] for k in NAMES], scale)
    assert torch.equal(out[0], plain[0]) and torch.equal(out[1], plain[1])
    _check(x, do, nb, P, T, c, Hq, Hkv, scale, out, grads)
    again = _run(x, do, P, T, c, scale)[1]
    assert all(torch.equal(a, b) for a, b in zip(grads, again))                    # additions in a fixed order


def test_sharp_weights():
    """Scores some tens apart: weights of nearly 1 and nearly 0, L far from 0."""
    P, T, c = [50], [200], 8
    x, do, nb = _case(7, P, T, c, 4, 2, spread=3.0)
    out, grads = _run(x, do, P, T, c, 0.2)
    _check(x, do, nb, P, T, c, 4, 2, 0.2, out, grads)


def test_long_items_are_cut_and_joined():
    """A prompt seen by so many rows that its keys' sums are made in pieces; and beacons, whose rows begin inside a tile."""
    P, T, c, Hq, Hkv = [140], [6000], 4, 4, 1
    x, do, nb = _case(8, P, T, c, Hq, Hkv)
    out, grads = _run(x, do, P, T, c, 1 / math.sqrt(D))
    _check(x, do, nb, P, T, c, Hq, Hkv, 1 / math.sqrt(D), out, grads)
    assert all(torch.equal(a, b) for a, b in zip(grads, _run(x, do, P, T, c, 1 / math.sqrt(D))[1]))


def test_many_trajectories_each_like_alone():
    """More items than blocks, every length different; a trajectory's gradients do not depend on its neighbours."""
    n, c, Hq, Hkv = 90, 8, 8, 4
    P, T = [(i * 37) % 150 for i in range(n)], [1 + (i * 53) % 170 for i in range(n)]
    x, do, nb = _case(9, P, T, c, Hq, Hkv)
    scale = 1 / math.sqrt(D)
    out, grads = _run(x, do, P, T, c, scale)
    _check(x, do, nb, P, T, c, Hq, Hkv, scale, out, grads, sequences=range(0, n, 11))
    for i in (3, 44, 89):
        cut = dict(prompt=slice(sum(P[:i]), sum(P[:i + 1])), tok=slice(sum(T[:i]), sum(T[:i + 1])), beacon=slice(sum(nb[:i]), sum(nb[:i + 1])))
        one = {k: x[k][cut[k.split("_")[0]]].contiguous() for k in NAMES}
        alone = _run(one, [do[0][cut["tok"]].contiguous(), do[1][cut["beacon"]].contiguous()], [P[i]], [T[i]], c, scale)[1]
        assert all(torch.equal(a, b[cut[k.split("_")[0]]]) for k, a, b in zip(NAMES, alone, grads))


def test_infinities_of_a_neighbour_do_not_spread():
    P, T, c, Hq, Hkv = [30, 50, 20], [70, 45, 100], 8, 6, 2
    x, do, nb = _case(10, P, T, c, Hq, Hkv)
    want = _run(x, do, P, T, c, 0.1)[1]
    mid = dict(prompt=slice(30, 80), tok=slice(70, 115), beacon=slice(8, 13))
    for k in NAMES:
        x[k][mid[k.split("_")[0]]] = float("inf") if k[-1] == "v" else float("nan")
    do[0][mid["tok"]] = float("nan")
    do[1][mid["beacon"]] = float("inf")
    got = _run(x, do, P, T, c, 0.1)[1]
    for k, a, b in zip(NAMES, want, got):
        keep = torch.ones(a.shape[0], dtype=torch.bool, device=DEV)
        keep[mid[k.split("_")[0]]] = False
        assert torch.equal(a[keep], b[keep]), k


def test_gradient_along_a_direction_against_differences():
    """The gradient's inner product with a direction against the change of the fp64 loss along it."""
    P, T, c, Hq, Hkv = [20], [50], 8, 2, 1
    x, do, nb = _case(11, P, T, c, Hq, Hkv)
    scale = 1 / math.sqrt(D)
    _, grads = _run(x, do, P, T, c, scale)
    rng = np.random.RandomState(3)
    dirs = {k: rng.randn(*x[k].shape) for k in NAMES}
    see = O.visible(20, 50, c)

    def loss(e):
        X = {k: f64(x[k]) + e * dirs[k] for k in NAMES}
        k, v = [np.concatenate([X["prompt_" + a][:, 0], X["beacon_" + a][:, 0], X["tok_" + a][:, 0]]) for a in "kv"]
        return sum((O.forward(see, np.concatenate([X["tok_q"][:, h], X["beacon_q"][:, h]]), k, v, scale)[1] *
                    np.concatenate([f64(do[0])[:, h], f64(do[1])[:, h]])).sum() for h in range(Hq))
    slope = (loss(1e-4) - loss(-1e-4)) / 2e-4
    got = sum((f64(g) * dirs[k]).sum() for k, g in zip(NAMES, grads))
    # every element is off by some 2^-8 of its terms with a sign of its own: their sum by that of the root of the squares
    assert abs(got - slope) <= 4 * 2.0 ** -8 * math.sqrt(sum(((f64(g) * dirs[k]) ** 2).sum() for k, g in zip(NAMES, grads))), (got, slope)


def test_waits_that_run_out_are_reported():
    P, T, c, Hq, Hkv = [300], [500], 8, 8, 2
    x, do, _ = _case(12, P, T, c, Hq, Hkv)
    want = _run(x, do, P, T, c, 0.1)[1]
    B.lib().bc_mask_attn_backward_set_wait_limit(1)
    try:
        with pytest.raises(B.BreadcrumbsError) as e:
            _run(x, do, P, T, c, 0.1)
        assert e.value.status == B.BC_ERR_TIMEOUT
    finally:
        B.lib().bc_mask_attn_backward_set_wait_limit(0)
    assert all(torch.equal(a, b) for a, b in zip(want, _run(x, do, P, T, c, 0.1)[1]))


def test_missing_prompt_and_beacon_arrays():
    x, do, _ = _case(13, [0], [10], 16, 4, 2)
    none = dict(x, prompt_k=None, prompt_v=None, beacon_q=None, beacon_k=None, beacon_v=None)
    ins = [none[k] for k in NAMES]
    out = B.bc_mask_attn_forward_lse([0], [10], 16, *ins, 0.1)
    got = B.bc_mask_attn_backward([0], [10], 16, *ins, out[0], None, out[2], None, do[0], None, 0.1)
    want = _run(x, do, [0], [10], 16, 0.1)[1]
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_binding_refuses_what_does_not_fit():
    P, T, c = [10], [20], 4
    x, do, _ = _case(14, P, T, c, 4, 2)
    ins = [x[k] for k in NAMES]
    out = B.bc_mask_attn_forward_lse(P, T, c, *ins, 0.1)
    ok = (P, T, c, *ins, *out, *do, 0.1)
    change = lambda i, v: ok[:i] + (v,) + ok[i + 1:]
    for bad in (change(0, [11]), change(1, [19]), change(2, 5), change(2, 0), change(0, [10, 0]), change(5, ins[2].float()), change(6, None),
                change(8, None), change(11, out[0][:, :3]), change(13, out[2].double()), change(15, None), change(17, 0.0), change(17, float("nan"))):
        with pytest.raises(B.BreadcrumbsError):
            B.bc_mask_attn_backward(*bad)
    with pytest.raises(B.BreadcrumbsError):
        B.bc_mask_attn_forward_lse(P, T, c, *[t[..., :64].contiguous() for t in ins], 0.1)
