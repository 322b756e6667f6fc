"""The training operators on arrays of more than 2^31 elements: the rows behind that border as the same rows in arrays of their own."""
import pytest
import torch

from paper_2510_13797_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16
BORDER = 2 ** 31


def _rand(g, *shape):
    x = torch.empty(shape, dtype=BF16, device=DEV)
    step = max(1, (1 << 27) // x[0].numel())
    for i in range(0, shape[0], step):                     # PyTorch's generator in 32-bit pieces
        x[i:i + step].normal_(generator=g)
    return x


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    yield
    torch.cuda.empty_cache()


def test_log_probabilities():
    n, vocab, last = 14700, 151936, 1000
    assert (n - last) * vocab < BORDER < (n - last // 2) * vocab
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x = _rand(g, n, vocab)
    t = torch.randint(0, vocab, (n,), generator=g, device=DEV)
    gl, ge = torch.randn(n, generator=g, device=DEV), torch.randn(n, generator=g, device=DEV)
    got = B.bc_token_logprobs(x, t, 10)
    grad = B.bc_token_logprobs_backward(x, t, got[2], got[1], gl, ge)
    tail, tt = x[-last:].clone(), t[-last:].clone()
    want = B.bc_token_logprobs(tail, tt, 10)
    assert all(torch.equal(a[-last:], b) for a, b in zip(got, want))
    assert torch.equal(grad[-last:], B.bc_token_logprobs_backward(tail, tt, want[2], want[1], gl[-last:].clone(), ge[-last:].clone()))


def test_norms_around_a_block():
    n, hidden, last = 262500, 8192, 700
    assert (n - last) * hidden < BORDER < (n - last // 2) * hidden
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    x, h = _rand(g, n, hidden), _rand(g, n, hidden)
    w = 1 + 0.1 * _rand(g, 2, hidden)
    ho, y = B.bc_block_norm(x, h, x, w[0], w[1], 1e-6, 0.5)
    dx, dh, dgate, _, _ = B.bc_block_norm_backward(x, ho, x, w[0], w[1], 1e-6, 0.5, True, y, h, weight_grads=False)
    cut = [a[-last:].clone() for a in (x, h, y)]
    want = B.bc_block_norm(cut[0], cut[1], cut[0], w[0], w[1], 1e-6, 0.5)
    assert torch.equal(ho[-last:], want[0]) and torch.equal(y[-last:], want[1])
    want = B.bc_block_norm_backward(cut[0], want[0], cut[0], w[0], w[1], 1e-6, 0.5, True, cut[2], cut[1], weight_grads=False)
    assert all(torch.equal(a[-last:], b) for a, b in zip((dx, dh, dgate), want))


def test_the_mask_forms_gradient():
    """Trajectories of 64 tokens: one tile of keys and one to two of queries, so nothing is cut into pieces."""
    n, T, c, heads, last = 16500, 64, 16, 16, 40
    nb = T // c
    assert BORDER < (n - last) * T * heads * 128
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    tok, bea = [[_rand(g, rows, heads, 128) for _ in range(4)] for rows in (n * T, n * nb)]
    args = (tok[0], tok[1], tok[2], bea[0], bea[1], bea[2])
    out = B.bc_mask_attn_forward_lse([0] * n, [T] * n, c, None, None, *args, 0.1)
    grads = B.bc_mask_attn_backward([0] * n, [T] * n, c, None, None, *args, *out, tok[3], bea[3], 0.1)[2:]
    end = lambda t: t[-last * (T if t.shape[0] == n * T else nb):].clone()
    some = [end(a) for a in args]
    want = B.bc_mask_attn_forward_lse([0] * last, [T] * last, c, None, None, *some, 0.1)
    assert all(torch.equal(end(a), b) for a, b in zip(out, want))
    want = B.bc_mask_attn_backward([0] * last, [T] * last, c, None, None, *some, *want, end(tok[3]), end(bea[3]), 0.1)[2:]
    assert all(torch.equal(end(a), b) for a, b in zip(grads, want))
