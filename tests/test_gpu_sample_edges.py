"""bc_sample where host threads, borders between elements, differences beyond the largest float or rows without a number could make
it go wrong, against its fp64 oracle (oracle/sampling_oracle.py): the tokens have to be equal."""
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


# Pairs (d, u) of fp32 numbers: in the row (-d, 0) the first element's share e^-d / (1 + e^-d) is u, off by 2^-42 to 2^-37 of it.  From an
# enumeration of the d whose weight lies about half-way between two powers of two.
BORDERS = [
    (0.3351668119430542, 0.4169839918613434), (0.3373848497867584, 0.41644486784935), (0.3393268287181854, 0.4159730076789856),
    (0.3422203063964844, 0.41527023911476135), (0.3429049551486969, 0.4151040017604828), (0.3438277244567871, 0.4148799777030945),
    (0.34420573711395264, 0.41478821635246277), (0.34737640619277954, 0.41401877999305725), (0.3482600748538971, 0.41380441188812256),
    (0.3515695333480835, 0.4130018651485443), (0.3532089293003082, 0.4126044809818268), (0.35387200117111206, 0.41244378685951233),
    (1.0292387008666992, 0.26323172450065613), (1.0367457866668701, 0.2617783844470978), (1.0469118356704712, 0.25981855392456055),
    (1.7248982191085815, 0.15124131739139557), (1.7295488119125366, 0.15064530074596405), (1.7386198043823242, 0.14948832988739014),
    (1.7453124523162842, 0.14863941073417664), (1.7517313957214355, 0.14782895147800446), (2.423910617828369, 0.08136747032403946),
    (2.4285147190093994, 0.08102399110794067), (2.4351704120635986, 0.08052979409694672), (0.3349699378013611, 0.417031854391098),
    (0.3350943624973297, 0.4170016050338745), (1.0195037126541138, 0.2651240825653076), (1.020089030265808, 0.2650100588798523),
    (1.7169504165649414, 0.15226438641548157), (1.7193050384521484, 0.15196070075035095), (2.4052348136901855, 0.08277438580989838),
    (2.4083049297332764, 0.08254159241914749),
]


def test_numbers_close_to_a_border_between_two_elements():
    """The weights are as good as their rounding to a multiple of 2^-45: a border is where fp64 puts it, to 2^-42 of itself."""
    d, u = np.array(BORDERS, dtype=np.float32).T
    p = 1.0 / (1.0 + np.exp(d.astype(np.float64)))
    off = np.abs(p / u.astype(np.float64) - 1)
    assert off.min() > 2.0 ** -42 and off.max() < 2.0 ** -37
    x = torch.zeros((len(d), 2), device=DEV)
    x[:, 0] = -torch.from_numpy(d).to(DEV)
    _check(x, u.tolist())
    _check(x, u.tolist(), p=[0.9999] * len(d))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_many_rows_of_a_full_vocabulary(dtype):
    """A batch that fills the device (fewer threads per block than a few rows get), every filter."""
    n, v = 20, 151936
    g = torch.Generator(device=DEV)
    g.manual_seed(33)
    x = torch.randn((n, v), generator=g, device=DEV) * 2.5
    x.scatter_add_(1, torch.randint(0, v, (n, 8), generator=g, device=DEV), 3 + 3 * torch.randn((n, 8), generator=g, device=DEV))
    x = x.to(dtype)
    u = torch.rand(n, generator=g, device=DEV).tolist()
    r = range(n)
    t = [[1.0, 0.7, 1.3, 0.05][i % 4] for i in r]
    _check(x, u, t=t)
    _check(x, u, t=t, p=[[0.95, 0.5, 0.99][i % 3] for i in r])
    _check(x, u, t=t, k=[[50, 1, 400, v, 5000][i % 5] for i in r], p=[[1.0, 0.9, 0.5][i % 3] for i in r])
