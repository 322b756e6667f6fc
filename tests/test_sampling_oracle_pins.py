"""Hand-worked cases of the sampling definition (oracle/sampling_oracle.py), and bc_sample's argument checks (no kernel runs)."""
import math

import numpy as np
import pytest

from oracle.sampling_oracle import kept, sample
from paper_2510_13797_b200 import binding as B

LN2 = math.log(2.0)


def test_running_mass_in_index_order():
    x = [0.0, LN2, 0.0]                      # weights 1/2, 1, 1/2 of the maximum: running mass 1/4, 3/4, 1
    assert [sample(x, u) for u in (0.0, 0.2499, 0.25, 0.7499, 0.75, 0.9999)] == [0, 0, 1, 1, 2, 2]


def test_filters_by_hand():
    x = [LN2, 2 * LN2, 0.0, 2 * LN2]         # weights 1/2, 1, 1/4, 1
    assert kept(x, top_k=1)[0].tolist() == [1]                      # the lower index of the two largest
    assert kept(x, top_k=3)[0].tolist() == [0, 1, 3]
    assert kept(x, top_p=1 / 2.75)[0].tolist() == [1]               # mass 1 of 2.75 is reached exactly by one element
    assert kept(x, top_p=1.01 / 2.75)[0].tolist() == [1, 3]
    assert kept(x, top_k=3, top_p=0.81)[0].tolist() == [0, 1, 3]    # 2 of 2.5 are 0.8: one more is needed
    assert kept(x, top_k=3, top_p=0.79)[0].tolist() == [1, 3]
    assert kept(x, min_p=0.4)[0].tolist() == [0, 1, 3]
    assert kept(x, min_p=7.0)[0].tolist() == [1, 3]                 # the maximum always stays
    assert kept(x, top_p=0.0)[0].tolist() == [1]
    assert kept(x, temperature=0.5)[1].tolist() == pytest.approx([0.25, 1, 1 / 16, 1])


def test_masked_and_degenerate_rows():
    inf = math.inf
    assert sample([-inf, 1.0, -inf], 0.9) == 1
    assert sample([-inf, -inf], 0.5) == 0
    assert sample([math.nan, 3.0, 3.0], 0.6) == 2
    assert [sample([1.0, inf, inf], u) for u in (0.4, 0.6)] == [1, 2]
    assert sample([1.0, 2.0, 2.0], 0.3, temperature=0.0) == 1
    assert sample([1.0, 2.0], math.nan, temperature=inf) == 0 and sample([1.0, 2.0], 1.0, temperature=inf) == 1


def test_frequencies_follow_the_distribution():
    x = np.log([0.1, 0.2, 0.3, 0.4])
    n = 10000                                # one uniform per cell of an even grid: counts are off by one at most
    got = np.bincount([sample(x, (i + 0.5) / n) for i in range(n)], minlength=4)
    assert np.all(np.abs(got - [1000, 2000, 3000, 4000]) <= 1)


def test_sample_refuses_bad_arguments():
    f = B.lib().bc_sample
    p = 1 << 20                              # never dereferenced: every call below is refused on the host
    ok = [p, 0, 100, 4, 100, None, None, None, None, p, p, None]
    for at, value, want in ((0, None, B.BC_ERR_INVALID_ARG), (9, None, B.BC_ERR_INVALID_ARG), (10, None, B.BC_ERR_INVALID_ARG),
                            (3, 0, B.BC_ERR_INVALID_ARG), (3, -1, B.BC_ERR_INVALID_ARG), (4, 0, B.BC_ERR_INVALID_ARG),
                            (2, 99, B.BC_ERR_INVALID_ARG), (0, p + 1, B.BC_ERR_INVALID_ARG), (5, p + 2, B.BC_ERR_INVALID_ARG),
                            (10, p + 4, B.BC_ERR_INVALID_ARG)):
        args = list(ok)
        args[at] = value
        assert f(*args) == want, (at, value)
    assert f(p, 0, 1 << 19, 1, (1 << 18) + 1, None, None, None, None, p, p, None) == B.BC_ERR_UNSUPPORTED
    assert f(p + 2, 1, 100, 4, 100, None, None, None, None, p, p, None) == B.BC_ERR_INVALID_ARG     # fp32 logits on a 2-byte boundary
