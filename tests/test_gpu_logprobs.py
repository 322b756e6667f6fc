"""bc_token_logprobs and its gradient against their fp64 definition (oracle/logprobs_oracle.py)."""
import numpy as np
import pytest
import torch

from oracle import logprobs_oracle as O
from paper_2510_13797_b200 import binding as B
from tests.harness import f64

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def _rows(seed, n, vocab, dtype, pad=0, spread=2.2):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn((n, vocab + pad), generator=g, device=DEV) * spread
    x = x.to(dtype)[:, :vocab]
    t = torch.randint(0, vocab, (n,), generator=g, device=DEV)
    return g, x, t


def _check(x, t, top_k, got, stats_too=True):
    """Differences to the maximum are exact or off by 2^-24 of themselves; a weight exp(d) is off by 2^-22 (the unit) and d * 2^-23 (its
    argument), which for the weights that count (d above -20) is under 3e-6; a sum has at most some hundred additions of 2^-24 in a
    row.  So ln s is off by 1e-5 at most, log p by that and 2^-23 of itself, the entropy by that relative to ln s and t / s."""
    logprob, entropy, stats, idx, top = got
    X, T = f64(x), t.cpu().numpy() if t is not None else np.full(x.shape[0], -1)
    for r in range(x.shape[0]):
        lp, H, (m, ls), order, want = O.logprobs(X[r], int(T[r]), top_k)
        if t is not None:
            g = float(logprob[r])
            assert g == lp or abs(g - lp) <= 1e-5 + 2.0 ** -23 * abs(lp), (r, g, lp)
        assert abs(float(entropy[r]) - H) <= 1e-5 * (1 + 2 * ls + H), (r, float(entropy[r]), H)
        assert float(stats[r, 0]) == m and abs(float(stats[r, 1]) - ls) <= 1e-5, (r, stats[r], m, ls)
        if top_k:
            assert np.array_equal(idx[r].cpu().numpy(), order), (r, idx[r].cpu().numpy(), order)
            z = f64(top[r])
            dead = want == -np.inf
            assert np.array_equal(z == -np.inf, dead) and np.all(np.abs(z[~dead] - want[~dead]) <= 1e-5 + 2.0 ** -23 * np.abs(want[~dead]))


@pytest.mark.parametrize("n,vocab,dtype,pad,top_k", [
    (1, 1, BF16, 0, 1), (3, 2, F32, 1, 2), (5, 7, BF16, 0, 7), (4, 13, F32, 0, 13), (2, 255, BF16, 2, 255), (9, 1000, BF16, 0, 100), (2, 2049, F32, 3, 256),
    (7, 4095, BF16, 1, 64), (3, 8192, BF16, 0, 256), (6, 8193, BF16, 6, 20), (65, 32000, BF16, 0, 5), (3, 50257, F32, 47, 50), (5, 50257, BF16, 0, 128),
    (4, 151936, BF16, 0, 100), (2, 262144, F32, 0, 256), (2, 262143, BF16, 0, 0), (1, 151936, F32, 5, 1)])
def test_forward_matches_the_definition(n, vocab, dtype, pad, top_k):
    _, x, t = _rows(vocab + n, n, vocab, dtype, pad)
    _check(x, t, top_k, B.bc_token_logprobs(x, t, top_k))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [5000, 40001])
def test_rows_where_the_alternatives_are_hard_to_find(vocab, dtype):
    """Many equal elements, sorted rows, the large ones all in a few threads' pieces, fewer elements with mass than alternatives."""
    _, x, t = _rows(3, 10, vocab, dtype)
    at = torch.arange(vocab, device=DEV)
    x[0] = 1.25
    x[1] = (at.float() / vocab * 20 - 10).to(dtype)
    x[2] = (10 - at.float() / vocab * 20).to(dtype)
    x[3] = torch.where((at // 8) % 256 < 30, x[3].abs() + 5, x[3])
    x[4] = float("-inf")
    x[4, 4000:4005] = torch.arange(5, device=DEV).to(dtype)
    x[5] = float("nan")
    x[5, 17] = -3.0
    x[6] = torch.where(at % 3 == 0, x[6], torch.full_like(x[6], float("nan")))
    x[7] = torch.where(at % 2 == 0, torch.zeros_like(x[7]), -torch.zeros_like(x[7]))    # 0 and -0 are equal
    x[8] = x[8] * 0 - 1e30
    x[9, 100:1500] = x[9].max()
    for k in (1, 100, 256):
        _check(x, t, k, B.bc_token_logprobs(x, t, k))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_infinities_and_rows_without_a_distribution(dtype):
    _, x, t = _rows(5, 8, 9001, dtype)
    inf = float("inf")
    x[0, [3, 8000]] = inf
    x[1] = -inf
    x[2] = float("nan")
    x[3] = torch.finfo(dtype).min
    x[4, :9000] = -inf
    x[5] = x[5] + 1e6 if dtype is F32 else x[5] * 1e4
    x[6, 5] = torch.finfo(dtype).max
    x[7] = x[7] - 3e4 if dtype is F32 else x[7] * 1e-30
    t[4], t[0], t[6] = 9000, 3, 4
    got = B.bc_token_logprobs(x, t, 20)
    _check(x, t, 20, got)
    g = torch.ones(8, device=DEV)
    grad = B.bc_token_logprobs_backward(x, t, got[2], got[1], g, g)
    assert torch.isfinite(grad).all() and not grad[1:4].any()
    _check_grad(x, t, g, g, grad)


def _check_grad(x, t, g, h, grad):
    X, T, G, H, got = f64(x), t.cpu().numpy(), f64(g), f64(h), f64(grad)
    for r in range(x.shape[0]):
        want, size = O.grad(X[r], int(T[r]), G[r], H[r])
        # one rounding to the gradient's type; p, log p and the entropy are off by 2e-5 of their terms at most (see _check); what is
        # below the smallest normal number may be flushed
        bound = torch.finfo(grad.dtype).eps / 2 * np.abs(want) + 4e-5 * size + 1e-37
        assert np.all(np.abs(got[r] - want) <= bound), (r, np.max(np.abs(got[r] - want) - bound))


@pytest.mark.parametrize("n,vocab,dtype,pad,shift", [
    (1, 1, BF16, 0, 0), (3, 5, F32, 0, 0), (5, 1001, BF16, 0, 0), (5, 1001, BF16, 7, 0), (6, 8191, F32, 1, 1), (2, 50257, BF16, 0, 3), (2, 50257, F32, 47, 0),
    (3, 151936, BF16, 0, 0), (3, 8192, BF16, 100, 1)])
def test_gradient_matches_the_formula(n, vocab, dtype, pad, shift):
    g, x, t = _rows(vocab, n, vocab + shift, dtype, pad)
    x, t = x[:, shift:], t.clamp(max=vocab - 1)              # rows that begin anywhere
    t[n // 2] = -100
    dl, de = torch.randn(n, generator=g, device=DEV), torch.randn(n, generator=g, device=DEV)
    _, entropy, stats, _, _ = B.bc_token_logprobs(x, t)
    grad = B.bc_token_logprobs_backward(x, t, stats, entropy, dl, de)
    _check_grad(x, t, dl, de, grad)
    zero = torch.zeros_like(dl)
    _check_grad(x, t, dl, zero, B.bc_token_logprobs_backward(x, t, stats, None, dl))
    _check_grad(x, t, zero, de, B.bc_token_logprobs_backward(x, None, stats, entropy, None, de))
    # into the caller's own rows: only the vocabulary's columns are written, wherever the rows begin
    for off in (0, 1, 8):
        wide = torch.full((n, vocab + 19), 7.0, dtype=dtype, device=DEV)
        B.bc_token_logprobs_backward(x, t, stats, entropy, dl, de, grad=wide[:, off:off + vocab])
        assert torch.equal(wide[:, off:off + vocab], grad) and (wide[:, :off] == 7).all() and (wide[:, off + vocab:] == 7).all()


def test_gradient_along_a_direction_against_differences_of_the_oracle():
    _, x, t = _rows(8, 3, 700, F32)
    dl, de = torch.tensor([0.5, -1.0, 2.0], device=DEV), torch.tensor([0.1, 0.3, -0.2], device=DEV)
    _, entropy, stats, _, _ = B.bc_token_logprobs(x, t)
    grad = f64(B.bc_token_logprobs_backward(x, t, stats, entropy, dl, de))
    d = np.random.RandomState(2).randn(3, 700)

    def loss(e):
        rows = [O.logprobs(f64(x)[r] + e * d[r], int(t[r]), 1) for r in range(3)]
        return sum(float(dl[r]) * rows[r][0] + float(de[r]) * rows[r][1] for r in range(3))
    # differences are exact to 1e-9 here, the kernel to 4e-5 of the terms (see _check_grad): 2100 terms of 0.01 on average
    assert abs((grad * d).sum() - (loss(1e-4) - loss(-1e-4)) / 2e-4) <= 4e-5 * np.abs(grad * d).sum() + 1e-6


def test_targets_outside_the_vocabulary_give_nothing():
    _, x, _ = _rows(9, 4, 300, BF16)
    t = torch.tensor([-1, 300, 1 << 40, -(1 << 40)], device=DEV)
    logprob, entropy, stats, _, _ = B.bc_token_logprobs(x, t)
    assert not logprob.any()
    one = torch.ones(4, device=DEV)
    assert not B.bc_token_logprobs_backward(x, t, stats, entropy, one).any()


def test_same_results_again_and_in_a_replayed_graph():
    g, x, t = _rows(10, 37, 30001, BF16)
    dl, de = torch.randn(37, generator=g, device=DEV), torch.randn(37, generator=g, device=DEV)

    def both():
        out = B.bc_token_logprobs(x, t, 64)
        return out + (B.bc_token_logprobs_backward(x, t, out[2], out[1], dl, de),)
    first = both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both()
    for _ in range(2):
        x.copy_(torch.randn(x.shape, generator=g, device=DEV))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(captured, both()))
    assert not torch.equal(captured[0], first[0])


def test_feeds_the_distillation_loss():
    """A teacher's hundred entries per position, as the loss takes them: distilling it into itself costs nothing but the mass left out."""
    n, vocab, k = 40, 5000, 100
    _, x, t = _rows(11, n, vocab, BF16, spread=4.0)
    _, _, _, idx, top = B.bc_token_logprobs(x, t, k)
    cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    loss, row_loss, _ = B.bc_distill_loss(cu, x, idx, top)
    assert float(row_loss.abs().max()) <= 2e-5          # log p of the stored entries against log q of the same row, both fp32


def test_binding_refuses_what_does_not_fit():
    _, x, t = _rows(12, 4, 100, BF16)
    bad = [lambda: B.bc_token_logprobs(x.half(), t), lambda: B.bc_token_logprobs(x, t.int()), lambda: B.bc_token_logprobs(x, t[:3]),
           lambda: B.bc_token_logprobs(x[0], t), lambda: B.bc_token_logprobs(x.t(), t), lambda: B.bc_token_logprobs(x, t, 101),
           lambda: B.bc_token_logprobs(x.cpu(), t), lambda: B.bc_token_logprobs_backward(x, t, None, None, torch.ones(4, device=DEV)),
           lambda: B.bc_token_logprobs_backward(x, t, torch.zeros((4, 2), device=DEV), None, torch.ones(4, device=DEV), torch.ones(4, device=DEV)),
           lambda: B.bc_token_logprobs_backward(x, t, torch.zeros((4, 2), device=DEV), None, torch.ones(4, device=DEV), grad=x.float())]
    for call in bad:
        with pytest.raises(B.BreadcrumbsError):
            call()
