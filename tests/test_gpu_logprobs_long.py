"""bc_token_logprobs where blocks note pieces of a long row for the alternatives: rows of their own for each block, and rows that two or
four blocks share; against sorting and summing in fp64 with PyTorch."""
import pytest
import torch

from paper_2510_13797_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def _fill(x, g):
    """Rows of every kind, so that each is met by several blocks at once: what is easy, and what leaves too many pieces."""
    n, vocab = x.shape
    at = torch.arange(vocab, device=DEV)
    up = (at.float() / vocab * 20 - 10).to(x.dtype)
    for r in range(n):
        kind = r % 12
        if kind == 1:
            x[r] = 1.25
        elif kind == 2:
            x[r] = up
        elif kind == 3:
            x[r] = up.flip(0)
        elif kind == 4:                                     # fewer elements with mass than alternatives
            x[r] = float("-inf")
            x[r, torch.randint(0, vocab, (30,), generator=g, device=DEV)] = 2.0
        elif kind == 5:
            x[r] = torch.where(at % 3 == 0, x[r], torch.full_like(x[r], float("nan")))
        elif kind == 6:                                     # the largest in the last pieces only
            x[r, -300:] += 20
        elif kind == 7:                                     # and in the first round only
            x[r, :300] += 20
        elif kind == 8:                                     # ties across the border of the alternatives
            x[r, torch.randint(0, vocab, (2000,), generator=g, device=DEV)] = 15.0
        elif kind == 9:
            x[r, torch.randint(0, vocab, (3,), generator=g, device=DEV)] = float("inf")
        elif kind == 10:
            x[r, torch.randint(0, vocab, (5,), generator=g, device=DEV)] = torch.finfo(x.dtype).max
        elif kind == 11:                                    # every piece of 8 has one of the large ones
            x[r, ::8] = x[r, ::8].abs() + 8


@pytest.mark.parametrize("n,vocab,dtype,pad,top_k", [
    (160, 40001, BF16, 0, 100), (152, 151936, BF16, 0, 20), (150, 50257, F32, 3, 128), (156, 70000, BF16, 1, 256), (149, 32000, F32, 0, 1),
    (96, 262144, BF16, 0, 100), (60, 262144, BF16, 0, 64), (84, 151936, F32, 0, 200), (48, 151937, F32, 2, 5)])
def test_long_rows(n, vocab, dtype, pad, top_k):
    g = torch.Generator(device=DEV)
    g.manual_seed(n + vocab)
    x = (torch.randn((n, vocab + pad), generator=g, device=DEV) * 2.2).to(dtype)[:, :vocab]
    _fill(x, g)
    t = torch.randint(0, vocab, (n,), generator=g, device=DEV)
    logprob, entropy, stats, idx, top = B.bc_token_logprobs(x, t, top_k)
    far = 2.0 ** 126
    for r in range(n):
        z = torch.where(x[r].isnan(), float("-inf"), x[r].double())
        order = torch.sort(z, descending=True, stable=True).indices[:top_k]
        assert torch.equal(idx[r].long(), order), r
        z = torch.where(z == float("-inf"), z, z.clamp(-far, far))
        m = z.max()
        d = z - m
        e = d.exp()
        ls = e.sum().log()
        lp = d - ls
        H = ls - (e * d.clamp(min=-1e4)).sum() / e.sum()
        # the bounds of test_gpu_logprobs.py: ln s within 1e-5, log p besides that within 2^-23 of itself
        near = lambda a, b: a == b or abs(a - b) <= 1e-5 + 2.0 ** -23 * abs(b)
        assert near(float(logprob[r]), float(lp[t[r]])), r
        assert float(stats[r, 0]) == float(m) and abs(float(stats[r, 1]) - float(ls)) <= 1e-5, r
        assert abs(float(entropy[r]) - float(H)) <= 1e-5 * (1 + 2 * float(ls) + float(H)), r
        got, want = top[r].double(), lp[order]
        assert bool(((got == want) | ((got - want).abs() <= 1e-5 + 2.0 ** -23 * want.abs())).all()), r
