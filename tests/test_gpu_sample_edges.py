"""bc_sample where host threads, differences beyond the largest float or rows without a number could make it go wrong, against its
fp64 oracle (oracle/sampling_oracle.py): the tokens have to be equal."""
import threading

import numpy as np
import pytest
import torch

from oracle.sampling_oracle import sample
from paper_2510_13797_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
INF, NAN = float("inf"), float("nan")


def _t(x, dtype=torch.float32):
    return None if x is None else torch.tensor(x, dtype=dtype, device=DEV)


def _check(x, u, t=None, k=None, p=None, floor=False):
    """floor: elements of less than 2^-46 of the largest weight, which are never chosen (breadcrumbs.h), are left out of the oracle's row."""
    n = len(x)
    got = B.bc_sample(x, _t(u), _t(t), _t(k, torch.int32), _t(p))
    rows = x.double().cpu().numpy()
    for r in range(n) if floor else ():
        rows[r][(rows[r] - rows[r].max()) / float(np.float32(t[r])) < -46 * np.log(2.0)] = -INF
    f32 = lambda v: [1.0] * n if v is None else [float(np.float32(a)) for a in v]
    t, p, k = f32(t), f32(p), [0] * n if k is None else k
    want = [sample(rows[r], np.float32(u[r]), t[r], k[r], p[r]) for r in range(n)]
    assert got.tolist() == want, [(r, g, w) for r, (g, w) in enumerate(zip(got.tolist(), want)) if g != w][:5]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_and_small_vocabularies_from_two_threads(dtype):
    """A call's shared memory follows its vocabulary: a thread that samples a small one must not take it from a thread that samples a
    large one."""
    n, sizes, f = 24, (151936, 500), B.lib().bc_sample
    inputs, failures = [], []
    for v in sizes:
        x = torch.randn((n, v), device=DEV).to(dtype)
        u = torch.rand(n, device=DEV)
        inputs.append((x, u, B.bc_sample(x, u), torch.cuda.Stream()))
    torch.cuda.synchronize()
    start = threading.Barrier(len(sizes))

    def work(x, u, want, stream):
        out, v = torch.empty_like(want), x.shape[1]
        args = (x.data_ptr(), int(dtype is torch.float32), v, n, v, None, None, None, None, u.data_ptr(), out.data_ptr(), stream.cuda_stream)
        torch.cuda.set_device(x.device)
        start.wait()
        try:
            status = {f(*args) for _ in range(20000)}      # as little else as possible between two calls, so that they overlap
            stream.synchronize()
            if status != {B.BC_OK} or not torch.equal(out, want):
                failures.append((v, status))
        except Exception as e:   # reported by the test's own thread
            failures.append(repr(e))

    threads = [threading.Thread(target=work, args=a) for a in inputs]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not failures


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("t", [1e37, 1e38, 3e38])
def test_lowest_value_as_a_mask_at_temperatures_that_reach_it(dtype, t):
    """Logits near 0 and the type's lowest value: differences of more than 3e38 that still weigh something."""
    n, v = 4, 2000
    g = torch.Generator(device=DEV)
    g.manual_seed(31)
    x = torch.full((n, v), torch.finfo(dtype).min, device=DEV, dtype=dtype)
    for r in range(n):
        at = torch.randperm(v, generator=g, device=DEV)[:500]
        x[r, at] = torch.randn(500, generator=g, device=DEV).to(dtype)
    x[2, 100], x[3, 100] = torch.finfo(dtype).max / 2, torch.finfo(dtype).max     # differences beyond the largest float
    for u in (0.0, 0.35, 0.7, 0.9999):
        us, ts = [u] * n, [t] * n
        _check(x, us, t=ts, floor=True)
        _check(x, us, t=ts, k=[600] * n, floor=True)
        _check(x, us, t=ts, k=[1999] * n, floor=True)
        _check(x, us, t=ts, p=[0.9] * n, floor=True)
        _check(x, us, t=ts, k=[600] * n, p=[0.99] * n, floor=True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_nan_and_minus_infinity_yield_their_first_element(dtype):
    n, v = 6, 4001
    x = torch.full((n, v), -INF, device=DEV, dtype=dtype)
    x[0, 0] = NAN
    x[1, :3999] = NAN
    x[2, 1:] = NAN
    x[3, 5] = NAN
    x[4, :] = NAN
    x[5, :600] = NAN
    for t in (None, [0.0] * n, [0.7] * n):
        _check(x, [0.5] * n, t=t)
        _check(x, [0.5] * n, t=t, k=[3] * n, p=[0.9] * n)
        assert B.bc_sample(x, torch.rand(n, device=DEV), _t(t)).tolist() == [0] * n
