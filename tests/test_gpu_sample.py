"""bc_sample against its fp64 oracle (oracle/sampling_oracle.py): the tokens have to be equal."""
import math

import numpy as np
import pytest
import torch

from oracle.sampling_oracle import sample
from paper_2510_13797_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF = float("inf")


def _check(logits, u, t=None, k=None, p=None, m=None, **kw):
    f = lambda x, d: None if x is None else torch.tensor(x, dtype=d, device=DEV)
    got = B.bc_sample(logits, f(u, torch.float32), f(t, torch.float32), f(k, torch.int32), f(p, torch.float32), f(m, torch.float32), **kw)
    x = logits.double().cpu().numpy()
    f32 = lambda v: [float(np.float32(a)) for a in v]
    n = len(x)
    t, p, m = [f32(v) if v is not None else d for v, d in ((t, [1.0] * n), (p, [1.0] * n), (m, [0.0] * n))]
    want = [sample(x[r], np.float32(u[r]), t[r], 0 if k is None else k[r], p[r] if p[r] == p[r] else 1.0, m[r] if m[r] == m[r] else 0.0) for r in range(n)]
    assert got.tolist() == want, [(r, g, w) for r, (g, w) in enumerate(zip(got.tolist(), want)) if g != w][:5]
    return got


def _logits(seed, n, v, dtype, pad=0, sigma=2.5):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn((n, v + pad), generator=g, device=DEV) * sigma
    x[:, :v].scatter_add_(1, torch.randint(0, v, (n, 8), generator=g, device=DEV), 3 + 3 * torch.randn((n, 8), generator=g, device=DEV))
    return x.to(dtype)[:, :v]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("v,pad", [(1, 0), (2, 5), (7, 0), (8, 0), (9, 0), (64, 3), (1000, 1), (4099, 0), (50257, 47), (151936, 0), (262144, 0)])
def test_vocabularies_strides_and_filters(dtype, v, pad):
    n = 24 if v < 100000 else 12
    x = _logits(v, n, v, dtype, pad)
    u = np.random.RandomState(v).rand(n).astype(np.float32)
    r = range(n)
    t = [[1.0, 0.7, 1.3, 0.05][i % 4] for i in r]
    k = [[0, 1, 5, 50, v, v + 7, 400, -3][i % 8] for i in r]
    p = [[1.0, 0.9, 0.5, 0.99, 0.0][i % 5] for i in r]
    m = [[0.0, 0.02, 0.3][i % 3] for i in r]
    _check(x, u)
    _check(x, u, t=t)
    _check(x, u, t=t, k=k)
    _check(x, u, t=t, p=p)
    _check(x, u, t=t, m=m)
    a = _check(x, u, t=t, k=k, p=p, m=m)
    b = _check(x, u, t=t, k=k, p=p, m=m)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ties_go_to_the_lowest_index(dtype):
    v = 20000
    x = torch.zeros((6, v), dtype=dtype, device=DEV)
    x[1, 5000:] = -1.0
    x[2] = torch.arange(v, device=DEV).remainder(7).to(dtype)
    x[3, ::3] = 0.5
    x[4, 1::2] = -0.0                                     # the two zeros are equal
    x[5, 10] = 3.0
    for u in (0.0, 0.25, 0.5, 0.999, 1 - 2.0 ** -24):
        us = [u] * 6
        _check(x, us, k=[100, 7000, 1, 6000, 10001, 2])
        _check(x, us, p=[0.5, 0.75, 0.3, 0.9, 0.25, 0.01])
        _check(x, us, k=[5000] * 6, p=[0.5, 0.75, 0.3, 0.9, 0.25, 0.01], m=[0.0, 0.9, 0.1, 1.0, 1.0, 0.5])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masked_lowest_and_infinite_logits(dtype):
    v, n = 5003, 12
    low = torch.finfo(dtype).min
    x = _logits(11, n, v, dtype).contiguous()
    x[0, :] = -INF
    x[1, :] = low
    x[2, 100:] = -INF
    x[3, 100:] = low
    x[4, 17], x[4, 4000] = INF, INF
    x[5, ::2] = float("nan")
    x[6, :] = float("nan")
    x[7, 3:] = -INF
    x[8, :-1] = -INF
    x[9, 0], x[9, 1] = torch.finfo(dtype).max, low
    x[10, :] = float("nan")
    x[10, 4999] = -5.0
    for u in (0.0, 0.3, 0.6, 0.99):
        us = [u] * n
        _check(x, us)
        _check(x, us, k=[50] * n)
        _check(x, us, p=[0.9] * n)
        _check(x, us, k=[2000] * n, p=[0.8] * n, m=[0.01] * n)


def test_extreme_parameters():
    v, n = 3001, 12
    x = _logits(12, n, v, torch.float32).contiguous()
    x[:, 7] = x[:, 1000] = x.amax(1)                       # equal maxima
    nan = float("nan")
    t = [0.0, -1.0, nan, 1e-30, 1e-45, INF, 1e30, 1e-3, 1.0, 1.0, 1.0, 100.0]
    for u in (0.0, 0.4, 0.7, 0.9999):
        us = [u] * n
        _check(x, us, t=t)
        _check(x, us, t=t, k=[3] * n)
        _check(x, us, t=t, p=[0.6] * n)
        _check(x, us, t=t, k=[1000] * n, p=[0.999] * n, m=[0.5] * n)
    _check(x, [nan, -1.0, 1.0, 2.0, INF, -INF] + [0.5] * 6)
    _check(x, [0.5] * n, p=[nan, -1.0, 0.0, 1e-30, 1 - 2.0 ** -24, 2.0, INF, -INF, 1.0, 0.5, 0.5, 0.5], m=[nan, -1.0, 2.0, INF, 1.0, 0.0] + [1e-38] * 6,
           k=[-2 ** 31, 2 ** 31 - 1, 0, 1] + [3000, 3001, 3002, 2] * 2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_infinite_temperature_over_the_whole_range(dtype):
    """Differences beyond the largest float, and a temperature that makes all of them nothing: every finite logit weighs the same."""
    n, v = 6, 1001
    x = _logits(13, n, v, torch.float32)
    x = (x / x.abs().amax() * 3.3e38).to(dtype)
    x[:, 5] = -INF
    x[0, :] = 3e38
    x[1, ::2] = -3e38
    for t in (INF, 3e38):
        for u in (0.0, 0.3, 0.9999):
            us, ts = [u] * n, [t] * n
            _check(x, us, t=ts)
            _check(x, us, t=ts, k=[300] * n)
            _check(x, us, t=ts, p=[0.6] * n)
            _check(x, us, t=ts, k=[600] * n, p=[0.7] * n)


def test_frequencies_of_a_stratified_uniform():
    """4096 rows of one distribution, one uniform per cell of an even grid: every token's count is its probability within one."""
    n, v = 4096, 37
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x = (torch.randn(v, generator=g, device=DEV)).expand(n, v).contiguous()
    u = (torch.arange(n, device=DEV, dtype=torch.float32) + 0.5) / n
    counts = torch.bincount(B.bc_sample(x, u), minlength=v).double()
    assert float((counts - torch.softmax(x[0].double(), 0) * n).abs().max()) <= 1.0


def test_output_stream_capture_and_agreement_with_argmax():
    n, v = 33, 151936
    x = _logits(21, n, v, torch.bfloat16)
    u = torch.rand(n, device=DEV)
    want = B.bc_sample(x, u, top_p=torch.full((n,), 0.9, device=DEV))
    out = torch.full((n + 3,), -1, dtype=torch.int64, device=DEV)
    top_p = torch.full((n,), 0.9, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    B.bc_sample(x, u, top_p=top_p, out=out[:n], stream=s)
    fresh = B.bc_sample(x, u, top_p=top_p, stream=s)
    s.synchronize()
    assert torch.equal(out[:n], want) and torch.equal(fresh, want) and out[n:].tolist() == [-1] * 3
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="thread_local"):
        B.bc_sample(x, u, top_p=top_p, out=out[:n])
    u.copy_(torch.rand(n, device=DEV))
    graph.replay()
    assert torch.equal(out[:n], B.bc_sample(x, u, top_p=top_p))
    best = torch.empty(n, dtype=torch.int64, device=DEV)
    B.bc_argmax(x.contiguous(), best)
    assert torch.equal(B.bc_sample(x, u, temperature=torch.zeros(n, device=DEV)), best)
    assert torch.equal(B.bc_sample(x, u, top_k=torch.ones(n, dtype=torch.int32, device=DEV)), best)


def test_binding_refuses_wrong_tensors():
    x, u = torch.zeros((4, 100), device=DEV), torch.zeros(4, device=DEV)
    for a in (dict(logits=x.double()), dict(logits=x.half()), dict(uniform=u.double()), dict(uniform=u[:3]), dict(top_k=u), dict(temperature=u.cpu()),
              dict(logits=x.t()), dict(logits=x[0]), dict(out=torch.zeros(4, dtype=torch.int32, device=DEV)), dict(logits=x[:, ::2])):
        with pytest.raises(B.BreadcrumbsError):
            B.bc_sample(**{**dict(logits=x, uniform=u), **a})
    with pytest.raises(B.BreadcrumbsError) as e:
        B.bc_sample(torch.zeros((1, 262145), device=DEV), u[:1])
    assert e.value.status == B.BC_ERR_UNSUPPORTED
