"""bc_block_norm and its gradient against their fp64 definition (oracle/block_norm_oracle.py)."""
import numpy as np
import pytest
import torch

from oracle import block_norm_oracle as O
from paper_2510_13797_b200 import binding as B
from tests.harness import f64, randn_bf16

pytestmark = pytest.mark.gpu
DEV = "cuda"
EPS = 1e-6
BF = 2.0 ** -8


def _inputs(seed, n, hidden, gate, weights=True):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rnd = lambda *s, scale=1.0: randn_bf16(g, s, DEV, scale=scale)
    gt = dict(none=lambda: None, vector=lambda: 1 + rnd(hidden, scale=0.3), rows=lambda: 1 + rnd(n, hidden, scale=0.3))[gate]()
    w1, w2 = [1 + rnd(hidden, scale=0.2) if weights else None for _ in range(2)]
    return rnd(n, hidden, scale=3.0), rnd(n, hidden, scale=2.0), gt, w1, w2, rnd(n, hidden), rnd(n, hidden)


def _f(t, like=1.0):
    return np.asarray(like) if t is None else f64(t)


SHAPES = [(1, 8, "none", True, True), (5, 8, "rows", False, True), (33, 24, "vector", True, True), (17, 256, "rows", True, False), (64, 264, "none", True, True),
          (7, 1000, "vector", False, True), (64, 1536, "rows", True, True), (300, 2048, "vector", True, True), (150, 4096, "none", False, False),
          (20, 4104, "vector", True, True), (31, 8192, "rows", True, True), (1, 8192, "vector", True, True), (700, 64, "vector", True, True)]


@pytest.mark.parametrize("n,hidden,gate,post,weights", SHAPES)
def test_forward_matches_the_definition(n, hidden, gate, post, weights):
    x, h, gt, w1, w2, _, _ = _inputs(n + hidden, n, hidden, gate, weights)
    scale = 0.7
    out, y = B.bc_block_norm(x, h, gt, w1, w2, EPS, scale, post)
    ref = O.stream(f64(x), f64(h), _f(gt), post, _f(w1), scale, EPS)
    # fp32: the mean's additions and a dozen operations of 2^-24, relative to the terms added; one rounding to bf16
    terms = np.abs(f64(h)) + np.abs(ref - f64(h))
    assert np.all(np.abs(f64(out) - ref) <= BF * np.abs(ref) + 2e-6 * terms)
    want = O.unit(f64(out), _f(w2), EPS)                      # the norm sees the stream as it is stored
    assert np.all(np.abs(f64(y) - want) <= (BF + 2e-6) * np.abs(want))
    again = B.bc_block_norm(x, h.clone(), gt, w1, w2, EPS, scale, post, want_y=False)
    assert torch.equal(again[0], out) and again[1] is None
    own = h.clone()
    B.bc_block_norm(x, own, gt, w1, w2, EPS, scale, post, h_out=own)    # in place
    assert torch.equal(own, out)


@pytest.mark.parametrize("n,hidden,gate,post,weights", SHAPES)
def test_gradient_matches_the_formula(n, hidden, gate, post, weights):
    x, h, gt, w1, w2, a, b = _inputs(n + hidden + 1, n, hidden, gate, weights)
    scale = 0.4
    h, _ = B.bc_block_norm(x, h, gt, w1, w2, EPS, scale, post)
    for da, db in ((a, b), (a, None), (None, b)):
        got = B.bc_block_norm_backward(x, h, gt, w1, w2, EPS, scale, post, da, db)
        z = np.zeros((n, hidden))
        args = (f64(x), f64(h), _f(gt), post, _f(w1), _f(w2), scale, EPS)
        dx, dh, dg, dp, dq = O.grad(*args, _f(da, z), _f(db, z))
        # the size of what is added up in each element: the row's means are sums in fp32 with 2^-24 an addition, some thirty in a row
        big = lambda t: np.abs(t).max(-1, keepdims=True)
        for name, mine, ref in (("dx", got[0], dx), ("dh", got[1], dh)):
            assert np.all(np.abs(f64(mine) - ref) <= BF * np.abs(ref) + 1e-5 * (big(ref) + 1e-30)), name
        if gate == "rows":
            assert np.all(np.abs(f64(got[2]) - dg) <= BF * np.abs(dg) + 1e-5 * big(dg))
        sums = [("pre", got[4], dq)] + ([("post", got[3], dp)] if post else []) + ([("gate", got[2], dg)] if gate == "vector" else [])
        for name, mine, ref in sums:                          # at most a few hundred additions in a row
            assert mine.dtype is torch.float32 and np.all(np.abs(f64(mine) - ref.sum(0)) <= 4e-5 * (np.abs(ref).sum(0).max() + 1e-30)), name
        assert (got[3] is None) == (not post) and (got[2] is None) == (gate == "none")
        again = B.bc_block_norm_backward(x, h, gt, w1, w2, EPS, scale, post, da, db)
        assert all(p is q or torch.equal(p, q) for p, q in zip(again, got))          # additions in a fixed order
        less = B.bc_block_norm_backward(x, h, gt, w1, w2, EPS, scale, post, da, db, weight_grads=False)
        assert torch.equal(less[0], got[0]) and torch.equal(less[1], got[1]) and less[3] is None and less[4] is None


def test_without_gate_norm_and_scale_it_is_the_plain_add_and_norm():
    x, h, _, _, w2, _, _ = _inputs(3, 65, 1536, "none")
    out, y = B.bc_block_norm(x, h, None, None, w2, EPS, 1.0, False)
    ho, yo = torch.empty_like(h), torch.empty_like(h)
    B.bc_add_rmsnorm(h, x, w2, EPS, ho, yo)
    assert torch.equal(out, ho)
    assert np.all(np.abs(f64(y) - f64(yo)) <= 2 * BF * np.abs(f64(yo)))              # both one rounding from the same value


def test_sums_over_many_rows_keep_their_precision():
    n, hidden = 40000, 64
    x, h, gt, w1, w2, a, b = _inputs(4, n, hidden, "vector")
    got = B.bc_block_norm_backward(x, h, gt, w1, w2, EPS, 1.0, True, a.abs(), b.abs())
    _, _, dg, dp, dq = O.grad(f64(x), f64(h), _f(gt), True, _f(w1), _f(w2), 1.0, EPS, f64(a.abs()), f64(b.abs()))
    for mine, ref in ((got[2], dg), (got[3], dp), (got[4], dq)):
        assert np.all(np.abs(f64(mine) - ref.sum(0)) <= 1e-5 * np.abs(ref).sum(0))


def test_rows_of_zeros_and_of_large_values():
    n, hidden = 6, 512
    x, h, gt, w1, w2, a, b = _inputs(5, n, hidden, "rows")
    x[0], h[1], x[2], h[2] = 0, 0, 0, 0
    x[3], h[4] = x[3] * 1e15, h[4] * 1e15                     # squares stay below the largest float
    out, y = B.bc_block_norm(x, h, gt, w1, w2, EPS, 1.0, True)
    ref = O.stream(f64(x), f64(h), f64(gt), True, f64(w1), 1.0, EPS)
    assert np.all(np.abs(f64(out) - ref) <= BF * np.abs(ref) + 2e-6 * (np.abs(f64(h)) + np.abs(ref - f64(h))))
    assert torch.isfinite(y).all() and not y[2].any()
    got = B.bc_block_norm_backward(x, out, gt, w1, w2, EPS, 1.0, True, a, b)
    want = O.grad(f64(x), f64(out), f64(gt), True, f64(w1), f64(w2), 1.0, EPS, f64(a), f64(b))
    for mine, r in zip(got[:3], want[:3]):
        assert torch.isfinite(mine).all()
        assert np.all(np.abs(f64(mine) - r) <= BF * np.abs(r) + 1e-5 * np.abs(r).max(-1, keepdims=True) + 1e-30)


def test_captured_and_replayed():
    x, h, gt, w1, w2, a, b = _inputs(6, 200, 1536, "vector")

    def both():
        o = B.bc_block_norm(x, h, gt, w1, w2, EPS, 0.5, True)
        return o + B.bc_block_norm_backward(x, o[0], gt, w1, w2, EPS, 0.5, True, a, b)
    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both()
    for scale in (1.0, 2.0):
        x.mul_(scale)
        graph.replay()
        assert all(torch.equal(p, q) for p, q in zip(captured, both()))


def test_binding_refuses_what_does_not_fit():
    x, h, gt, w1, w2, a, b = _inputs(7, 4, 64, "rows")
    bad = [lambda: B.bc_block_norm(x.float(), h, gt, w1, w2, EPS), lambda: B.bc_block_norm(x, h[:3], gt, w1, w2, EPS),
           lambda: B.bc_block_norm(x, h, gt[:2], w1, w2, EPS), lambda: B.bc_block_norm(x, h, gt, w1[:8], w2, EPS),
           lambda: B.bc_block_norm(x.t(), h, gt, w1, w2, EPS), lambda: B.bc_block_norm(x, None, gt, w1, w2, EPS), lambda: B.bc_block_norm(x[:0], h[:0], None, w1, w2, EPS),
           lambda: B.bc_block_norm(x[:, :60].contiguous(), h[:, :60].contiguous(), None, None, None, EPS),
           lambda: B.bc_block_norm_backward(x, h, gt, w1, w2, EPS, 1.0, True, None, None), lambda: B.bc_block_norm_backward(x, h, gt, w1, w2, EPS, 1.0, True, a, b[:1])]
    for call in bad:
        with pytest.raises(B.BreadcrumbsError):
            call()


@pytest.mark.parametrize("n,hidden", [(700, 1536), (400, 4096), (200, 8192)])
def test_the_streams_gradient_in_place(n, hidden):
    """dh may be dh_out itself; rows of several rounds."""
    x, h, gt, w1, w2, a, b = _inputs(n, n, hidden, "rows")
    want = B.bc_block_norm_backward(x, h, gt, w1, w2, EPS, 0.5, True, a, b, weight_grads=False)
    dx, dgate = torch.empty_like(x), torch.empty_like(x)
    status = B.lib().bc_block_norm_backward(n, hidden, x.data_ptr(), h.data_ptr(), gt.data_ptr(), hidden, 1, w1.data_ptr(), w2.data_ptr(), 0.5, EPS,
                                            a.data_ptr(), b.data_ptr(), dx.data_ptr(), a.data_ptr(), dgate.data_ptr(), None, None, None, 0,
                                            torch.cuda.current_stream().cuda_stream)
    assert status == B.BC_OK
    assert torch.equal(dx, want[0]) and torch.equal(a, want[1]) and torch.equal(dgate, want[2])


def test_two_graphs_of_the_gradient():
    """Each with a workspace of its own, replayed by turns and at once."""
    x, h, gt, w1, w2, a, b = _inputs(77, 900, 512, "vector")
    call = lambda: B.bc_block_norm_backward(x, h, gt, w1, w2, EPS, 0.5, True, a, b)
    want = call()
    graphs, got, streams = [torch.cuda.CUDAGraph() for _ in range(2)], [], [torch.cuda.Stream() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph):
            got.append(call())
    for _ in range(5):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(t, w) for out in got for t, w in zip(out, want))
