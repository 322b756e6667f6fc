"""bc_chunk_attn and bc_prefill_chunk against the fp64 oracle (oracle/chunk_oracle.py over the cache's oracle)."""
import math

import numpy as np
import pytest
import torch

from oracle.breadcrumbs_oracle import SeqCache
from oracle.chunk_oracle import chunk_attend
from oracle.norm_rope_oracle import norm_rope_split
from oracle.paging_model import OK
from oracle.sampling_oracle import sample
from paper_2510_13797_b200 import binding as B
from tests.harness import Pair, f64, randn_bf16

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _i32(xs):
    return torch.tensor(list(xs), dtype=torch.int32, device=DEV)


def _cu(ms):
    return _i32(np.concatenate([[0], np.cumsum(ms)]))


def _assert_chunk(out, ref, mag, f32=False):
    """The softmax weights are rounded to bf16 for the second product (2^-8 each, so 2^-8 of sum w |V|) and the result once more;
    fp32 scores of up to 128 products are off by some 1e-5, and with them the weights: 1e-4 of sum w |V| covers the fp32 part."""
    assert tuple(out.shape) == ref.shape
    if ref.size == 0:
        return
    err = np.abs(f64(out) - ref) - ((0.0 if f32 else 2.0 ** -8) * np.abs(ref) + (2.0 ** -8 + 1e-4) * mag + 1e-30)
    assert err.max() <= 0, f"{err.max():.3e} over the bound at {np.unravel_index(err.argmax(), err.shape)}"


def _cache(Hkv, G, D, ps, c, plens, gens, seed, L=1, flags=0, slots=None):
    """A pair (library and oracle) with stored prompts and gens[i] generated tokens (with their beacons).  The pool starts as NaNs:
    rows that hold no entry must not matter."""
    n = len(plens)
    slots = list(range(n)) if slots is None else slots
    pages = lambda p, t: -(-p // ps) + (-(-(t // c) // ps) + -(-min(c, t) // ps) if c > 1 else -(-t // ps)) + 2
    per = max(pages(p, t) for p, t in zip(plens, gens))
    pair = Pair(L, Hkv, Hkv * G, D, ps, max_seqs=max(slots) + 2, num_pages=sum(pages(p, t) for p, t in zip(plens, gens)), max_pages_per_seq=per,
                c_default=c, flags=flags)
    pair.gpu.pool.fill_(255)
    g = _gen(seed)
    assert pair.open(slots, plens) == [OK] * n
    nb = sum(t // c for t in gens) if c > 1 else 0
    for l in range(L):
        pair.prefill(l, slots, plens, randn_bf16(g, (sum(plens), Hkv, D), DEV), randn_bf16(g, (sum(plens), Hkv, D), DEV))
        if sum(gens):
            assert pair.restore(l, slots, gens, *[randn_bf16(g, (x, Hkv, D), DEV) for x in (sum(gens), sum(gens), max(nb, 1), max(nb, 1))]) == [OK] * n
    return pair, slots, g


def _run(pair, slots, ms, g, first=None, layer=0, scale=None):
    """One call on the library and on the oracle; guard rows behind the last query stay untouched."""
    total, Hq, D = sum(ms), pair.Hq, pair.D
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    q = randn_bf16(g, (total, Hq, D), DEV)
    out = torch.full((total + 3, Hq, D), 7.0, dtype=pair.gpu.out_dtype, device=DEV)
    pair.gpu.bc_chunk_attn(layer, _i32(slots), _cu(ms), total, q, out[:total], scale, None if first is None else _i32(first))
    torch.cuda.synchronize()
    assert float(out[total:].min()) == 7.0 == float(out[total:].max())
    ref, mag, a = [], [], 0
    for i, s in enumerate(slots):
        K, V = pair.seqs[s].entries(layer) if s in pair.seqs else (np.zeros((0, pair.Hkv, D)),) * 2
        f = K.shape[0] - ms[i] if first is None else first[i]
        r, m = chunk_attend(f64(q)[a:a + ms[i]], K, V, f, scale)
        ref.append(r); mag.append(m)
        a += ms[i]
    _assert_chunk(out[:total], np.concatenate(ref), np.concatenate(mag), f32=pair.gpu.out_dtype == torch.float32)
    assert pair.gpu.bc_poll_error()[0] == 0
    return q, out[:total]


REF = B.BC_FLAG_ATTN_REFERENCE
CASES = [  # Hkv, G, D, page, c, prompts, generated, chunk lengths
    (2, 6, 128, 16, 1, [40, 200, 1, 129], [0, 0, 0, 0], [40, 7, 1, 129]),
    (8, 4, 128, 16, 16, [70, 300, 0, 16], [37, 16 * 9 + 5, 5, 16 * 3 + 15], [3, 5, 5, 15]),
    (1, 16, 64, 16, 4, [33, 500], [4 * 70 + 3, 7], [2, 1]),
    (2, 7, 64, 24, 1, [0, 511, 97], [30, 1, 0], [30, 1, 50]),
    (4, 1, 128, 5, 8, [129, 3, 260], [8 * 20 + 7, 8 * 2 + 1, 8 * 140 + 6], [7, 1, 6]),
    (1, 1, 64, 1, 1, [300, 20], [0, 0], [256, 0]),
    (2, 3, 128, 128, 32, [127, 128, 129], [32 * 130 + 31, 31, 32 * 5 + 20], [31, 31, 20]),
    (8, 2, 64, 64, 3, [1, 0, 65], [3 * 9 + 2, 2, 1], [2, 1, 1]),
    (1, 5, 128, 6, 2, [400], [2 * 33 + 1], [1]),
]


@pytest.mark.parametrize("flags", [REF, 0, B.BC_FLAG_OUT_F32, B.BC_FLAG_DEBUG_BOUNDS])
@pytest.mark.parametrize("Hkv,G,D,ps,c,plens,gens,ms", CASES)
def test_last_entries_match_oracle(Hkv, G, D, ps, c, plens, gens, ms, flags):
    pair, slots, g = _cache(Hkv, G, D, ps, c, plens, gens, seed=5, flags=flags)
    _run(pair, slots, ms, g)
    pair.check_state()


@pytest.mark.parametrize("ctas", [0, 1, 3, 40, 304])
@pytest.mark.parametrize("Hkv,G,D,ps,c,plens,gens,ms", [
    (2, 6, 128, 16, 1, [1500, 700, 0, 64], [20, 0, 9, 64], [11, 300, 9, 0]),
    (1, 4, 64, 8, 16, [900, 5, 1300], [16 * 40 + 9, 16 * 300 + 3, 11], [9, 3, 11]),
])
def test_spans_of_any_number_of_blocks(Hkv, G, D, ps, c, plens, gens, ms, ctas):
    pair, slots, g = _cache(Hkv, G, D, ps, c, plens, gens, seed=6)
    pair.gpu.bc_set_attn_ctas(ctas)
    for _ in range(3):                                     # the second and third call find the first one's scratch
        _run(pair, slots, ms, g)


@pytest.mark.parametrize("Hkv,G,D", [(2, 6, 128), (1, 3, 64)])
@pytest.mark.parametrize("ps", [2, 3, 4, 8, 12, 20, 40])
def test_page_sizes(Hkv, G, D, ps):
    """Tensor copies of 4 to 8 entries and copies row by row, across the three segments."""
    pair, slots, g = _cache(Hkv, G, D, ps, 3, [70, 201, 0], [3 * 30 + 2, 1, 3 * 25], seed=21)
    _run(pair, slots, [50, 90, 25], g)
    _run(pair, slots, [1, 2, 0], g)


def test_one_sequence_several_times_and_units_of_one_group():
    """Items of the same sequence, lengths that leave a second group of rows empty, full or with one token."""
    # a group: 32 tokens, a unit: 64; a call has at most as many items as the cache has slots
    pair, slots, g = _cache(2, 4, 128, 16, 1, [400, 90], [0, 0], seed=22, slots=[0, 40])
    _run(pair, [0, 40, 0, 0, 40, 0], [31, 33, 32, 65, 64, 1], g, first=[100, 3, 300, 335, 26, 399])
    _run(pair, [0] * 40, [1, 34] * 20, g, first=[9 * i for i in range(40)])


def test_two_caches_on_two_streams_at_once():
    caches = [_cache(2, 6, 128, 16, 1, [700, 40], [0, 0], seed=23), _cache(1, 4, 64, 16, 4, [300], [4 * 50 + 3], seed=24)]
    calls = []
    for pair, slots, g in caches:
        n = 130 if len(slots) == 2 else 3
        ms = [n, 20][:len(slots)]
        q = randn_bf16(g, (sum(ms), pair.Hq, pair.D), DEV)
        alone, out = torch.empty_like(q), torch.empty_like(q)
        args = (0, _i32(slots), _cu(ms), sum(ms), q)
        pair.gpu.bc_chunk_attn(*args, alone, 0.1)
        calls.append((pair, args, alone, out, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for pair, args, _, out, s in calls:
            pair.gpu.bc_chunk_attn(*args, out, 0.1, stream=s)
    torch.cuda.synchronize()
    for pair, _, alone, out, _ in calls:
        assert torch.equal(alone, out)
        assert pair.gpu.bc_poll_error()[0] == 0


@pytest.mark.parametrize("ctas", [0, 64, 304])
def test_one_long_cache_between_many_short_ones(ctas):
    """Spans much shorter than the longest unit: a unit in many more pieces than are joined at once, between units that are not cut."""
    plens = [40] * 30 + [30000] + [40] * 41
    pair, slots, g = _cache(4, 2, 64, 16, 1, plens, [0] * len(plens), seed=21)
    pair.gpu.bc_set_attn_ctas(ctas)
    for ms in ([1] * len(plens), [1 + i % 3 for i in range(len(plens))]):
        _run(pair, slots, ms, g)


def test_few_units_in_many_pieces():
    """Fewer units than thread blocks: one sequence over hundreds of key tiles, few rows and many."""
    pair, slots, g = _cache(1, 6, 128, 16, 1, [40000], [0], seed=22)
    _run(pair, slots, [1], g)
    _run(pair, slots, [30], g)
    _run(pair, slots, [7], g, first=[20000])


def test_results_do_not_change_from_call_to_call():
    pair, slots, g = _cache(2, 6, 128, 16, 1, [5000, 1200], [40, 10], seed=7)
    q, out = _run(pair, slots, [33, 10], g)
    for _ in range(5):
        again = torch.empty_like(out)
        pair.gpu.bc_chunk_attn(0, _i32(slots), _cu([33, 10]), 43, q, again, 1 / math.sqrt(128))
        assert torch.equal(again, out)


@pytest.mark.parametrize("flags", [REF, 0])
def test_first_past_the_ends_and_rows_that_see_nothing(flags):
    pair, slots, g = _cache(2, 4, 128, 16, 4, [50, 0, 20, 8], [4 * 3 + 2, 0, 4, 0], seed=8, flags=flags)
    _run(pair, slots, [9, 3, 5, 150], g, first=[-4, 0, 1000, -100])
    _run(pair, [1, 0], [0, 1], g, first=[5, -1])
    _run(pair, [0, 1, 4, -7, 99], [2, 1, 3, 2, 1], g)        # slots that are not open, or not there: zeros
    _run(pair, slots, [1, 1, 1, 1], g, first=[2 ** 31 - 1, -2 ** 31, 3, 0])


def test_layers_and_batch_order():
    pair, slots, g = _cache(2, 2, 64, 16, 4, [100, 30, 77], [9, 4, 3], seed=9, L=3)
    for l in (2, 0, 1):
        _run(pair, [2, 0, 1], [3, 1, 2], g, layer=l)
        _run(pair, [1], [1], g, layer=l, scale=0.5)


@pytest.mark.parametrize("n", [300, 512])
def test_many_items(n):
    rng = np.random.RandomState(n)
    plens = rng.randint(0, 60, size=n).tolist()
    ms = [int(rng.randint(0, p + 1)) if i % 3 else min(p, 1) for i, p in enumerate(plens)]
    ms[5], plens[5] = 200, 400
    pair, slots, g = _cache(1, 4, 64, 16, 1, plens, [0] * n, seed=10)
    _run(pair, slots, ms, g)


def test_many_long_chunks():
    """More items with many query tiles than one pass counts together, at 8 tokens per tile."""
    n = 70
    plens = [90 + i for i in range(n)]
    pair, slots, g = _cache(1, 16, 64, 16, 1, plens, [0] * n, seed=11)
    _run(pair, slots, [80 + (i % 11) for i in range(n)], g)


def test_values_of_other_rows_do_not_spread():
    """A NaN query spoils its own rows; a sequence with NaN entries spoils no other."""
    Hkv, G, D = 2, 6, 128
    pair, slots, g = _cache(Hkv, G, D, 16, 1, [70, 90], [0, 0], seed=12)
    q, out = _run(pair, slots, [30, 40], g)
    q2 = q.clone()
    q2[10, 3] = float("nan")
    k = randn_bf16(g, (90, Hkv, D), DEV)
    k[50] = float("nan")
    pair.gpu.bc_prefill(0, _i32([1]), _cu([90]), 90, k, k)
    out2 = torch.empty_like(out)
    pair.gpu.bc_chunk_attn(0, _i32(slots), _cu([30, 40]), 70, q2, out2, 1 / math.sqrt(D))
    assert bool(out2[10, 3].isnan().all()) and bool(out2[30:].isnan().any())
    keep = torch.ones((30, Hkv * G), dtype=torch.bool, device=DEV)
    keep[10, 3] = False
    assert torch.equal(out2[:30][keep], out[:30][keep])


@pytest.mark.parametrize("flags", [REF, 0])
@pytest.mark.parametrize("Hkv,G,D,ps,plens,step", [(2, 6, 128, 16, [300, 5, 131], 100), (1, 7, 64, 24, [260, 64, 0], 33), (8, 4, 128, 16, [97, 1], 1),
                                                  (1, 1, 128, 7, [80, 40], 27)])
def test_prompts_in_chunks(Hkv, G, D, ps, plens, step, flags):
    """A ragged batch of prompts, `step` tokens at a time: outputs of every chunk, the stored entries, the rest of the pool untouched."""
    if step == 1:
        plens = [min(p, 6) for p in plens]
    n, L = len(plens), 2
    pair = Pair(L, Hkv, Hkv * G, D, ps, max_seqs=n + 1, num_pages=sum(-(-p // ps) for p in plens) + 2, max_pages_per_seq=max(plens) // ps + 2, flags=flags)
    pair.gpu.pool.fill_(255)
    slots = list(range(n))
    assert pair.open(slots, plens) == [OK] * n
    g = _gen(13)
    K = [[randn_bf16(g, (p, Hkv, D), DEV) for p in plens] for _ in range(L)]
    V = [[randn_bf16(g, (p, Hkv, D), DEV) for p in plens] for _ in range(L)]
    scale = 1 / math.sqrt(D)
    for at in range(0, max(plens), step):
        ms = [max(0, min(step, p - at)) for p in plens]
        total, first = sum(ms), [min(at, p) for p in plens]
        for l in range(L):
            q = randn_bf16(g, (total, Hkv * G, D), DEV)
            new = lambda X: torch.cat([x[f:f + m] for x, f, m in zip(X[l], first, ms)])
            out = torch.empty((total, Hkv * G, D), dtype=torch.bfloat16, device=DEV)
            pair.gpu.bc_prefill_chunk(l, _i32(slots), _i32(first), _cu(ms), total, q, new(K), new(V), out, scale)
            parts = [chunk_attend(f64(x), f64(K[l][i][:f + m]), f64(V[l][i][:f + m]), f, scale)
                     for i, (x, f, m) in enumerate(zip(q.split(ms), first, ms))]
            _assert_chunk(out, np.concatenate([p[0] for p in parts]), np.concatenate([p[1] for p in parts]))
    for l in range(L):
        for i, p in enumerate(plens):
            if p:
                k, v = pair.gpu.bc_export_seq(l, i, p)
                assert torch.equal(k, K[l][i]) and torch.equal(v, V[l][i])
    used = sum(-(-p // ps) for p in plens) * ps * 2 * Hkv * D * 2
    assert int(pair.gpu.pool.view(L, -1)[:, used:].min()) == 255          # pages that belong to no prompt
    pair.check_state()


def test_prefill_chunk_past_the_prompt_is_not_stored():
    Hkv, G, D = 2, 2, 64
    pair, slots, g = _cache(Hkv, G, D, 16, 1, [20, 40], [0, 0], seed=14)
    before = pair.gpu.pool.clone()
    new = randn_bf16(g, (12, Hkv, D), DEV)
    q, out = randn_bf16(g, (12, Hkv * G, D), DEV), torch.empty((12, Hkv * G, D), dtype=torch.bfloat16, device=DEV)
    pair.gpu.bc_prefill_chunk(0, _i32([0, 1, 2]), _i32([20, -6, 0]), _cu([5, 6, 1]), 12, q, new, new, out, 0.1)
    assert torch.equal(pair.gpu.pool, before)
    K, V = pair.seqs[0].entries(0)
    ref, mag = chunk_attend(f64(q)[:5], K, V, 20, 0.1)
    _assert_chunk(out[:5], ref, mag)
    assert float(out[5:].abs().max()) == 0.0                              # rows that see nothing; a slot that is not open
    assert pair.gpu.bc_poll_error()[0] == 0


def test_pages_beyond_four_gigabytes():
    Hkv, G, D, ps, far = 8, 4, 128, 16, 1_100_000
    cache = B.Cache(1, Hkv, Hkv * G, D, 1, ps, 2, far // ps + 80, far // ps + 1)
    slots = _i32([0, 1])
    cache.bc_seq_open(slots, _i32([far, 700]))                            # slot 0 takes the first 4.5 GB, slot 1's pages lie behind
    g = _gen(15)
    k, v = [randn_bf16(g, (700, Hkv, D), DEV) for _ in range(2)]
    q, out = randn_bf16(g, (65, Hkv * G, D), DEV), torch.empty((65, Hkv * G, D), dtype=torch.bfloat16, device=DEV)
    cache.bc_prefill(0, slots[1:], _cu([635]), 635, k[:635].contiguous(), v[:635].contiguous())
    cache.bc_prefill_chunk(0, slots[1:], _i32([635]), _cu([65]), 65, q, k[635:].contiguous(), v[635:].contiguous(), out, 0.09)
    ref, mag = chunk_attend(f64(q), f64(k), f64(v), 635, 0.09)
    _assert_chunk(out, ref, mag)
    assert cache.bc_get_state(1)["prompt_pages"][0] * ps * 2 * Hkv * D * 2 > 1 << 32


def test_between_steps_on_another_stream_and_captured():
    """Chunk calls between the steps of a decode loop, on a stream of their own, and replayed from a graph: the steps' results and the
    chunks' are those of the plain order."""
    Hkv, G, D, c = 2, 6, 128, 4
    scale = 1 / math.sqrt(D)
    pair, slots, g = _cache(Hkv, G, D, 16, c, [90, 33, 260], [0, 0, 0], seed=16)
    n, sl = 3, _i32([0, 1, 2])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for t in range(1, 10):
        q, k, v = [randn_bf16(g, (n, h, D), DEV) for h in (Hkv * G, Hkv, Hkv)]
        torch.cuda.current_stream().wait_stream(s)
        _, out, ref = pair.step(0, slots, q, k, v, scale)
        w = pair.model.state(0)["window_len"]
        again = torch.empty((n, Hkv * G, D), dtype=torch.bfloat16, device=DEV)
        s.wait_stream(torch.cuda.current_stream())
        pair.gpu.bc_chunk_attn(0, sl, _cu([1] * n), n, q, again, scale, stream=s)
        s.synchronize()
        for i in range(n):
            K, V = pair.seqs[i].entries(0)
            r, m = chunk_attend(f64(q)[i:i + 1], K, V, K.shape[0] - 1, scale)
            _assert_chunk(again[i:i + 1], r, m)
            _assert_chunk(out[i:i + 1], r, m)
        if w == c:
            pair.compress(0, slots, randn_bf16(g, (n, Hkv, D), DEV), randn_bf16(g, (n, Hkv, D), DEV))
            s.wait_stream(torch.cuda.current_stream())
    pair.check_state()
    ms = [5, 2, 1]
    q, out = randn_bf16(g, (8, Hkv * G, D), DEV), torch.zeros((8, Hkv * G, D), dtype=torch.bfloat16, device=DEV)
    cu = _cu(ms)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="thread_local"):
        pair.gpu.bc_chunk_attn(0, sl, cu, 8, q, out, scale)
    for _ in range(3):
        q.copy_(randn_bf16(g, q.shape, DEV))
        cu.copy_(_cu(ms))
        graph.replay()
        torch.cuda.synchronize()
        a = 0
        for i, m in enumerate(ms):
            K, V = pair.seqs[i].entries(0)
            r, mag = chunk_attend(f64(q)[a:a + m], K, V, K.shape[0] - m, scale)
            _assert_chunk(out[a:a + m], r, mag)
            a += m
        ms = ms[1:] + ms[:1]                                   # lengths are read on the device: the graph follows them
        pair.append(0, slots, randn_bf16(g, (n, Hkv, D), DEV), randn_bf16(g, (n, Hkv, D), DEV))


def test_a_wait_that_runs_out_is_reported_and_leaves_the_cache_usable():
    pair, slots, g = _cache(2, 4, 128, 16, 1, [900, 400], [0, 0], seed=17)
    q, out = randn_bf16(g, (50, 8, 128), DEV), torch.empty((50, 8, 128), dtype=torch.bfloat16, device=DEV)
    pair.gpu.bc_set_wait_limit(1)
    pair.gpu.bc_chunk_attn(0, _i32(slots), _cu([30, 20]), 50, q, out, 0.1)
    assert pair.gpu.bc_poll_error()[0] == B.BC_ERR_TIMEOUT
    pair.gpu.bc_set_wait_limit(0)
    pair.gpu.bc_clear_error()
    _run(pair, slots, [30, 20], g)


def test_refusals():
    cache = B.Cache(2, 2, 4, 64, 1, 16, max_seqs=4, num_pages=8, max_pages_per_seq=2)
    sl, cu, f = _i32([0, 1]), _cu([1, 1]), _i32([0, 0])
    q, kv = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device=DEV), torch.zeros((2, 2, 64), dtype=torch.bfloat16, device=DEV)
    out = torch.full_like(q, 7.0)
    chunk = lambda **a: cache.bc_chunk_attn(**{**dict(layer=0, slots=sl, cu_q=cu, total_q=2, q=q, out=out, sm_scale=1.0), **a})
    fill = lambda **a: cache.bc_prefill_chunk(**{**dict(layer=0, slots=sl, first=f, cu_chunk=cu, total=2, q=q, k=kv, v=kv, out=out, sm_scale=1.0), **a})
    for call, bad in ((chunk, dict(layer=2)), (chunk, dict(layer=-1)), (chunk, dict(sm_scale=0.0)), (chunk, dict(sm_scale=-1.0)), (chunk, dict(total_q=3)),
                      (chunk, dict(q=q.float())), (chunk, dict(out=out.float())), (chunk, dict(cu_q=cu.long())), (chunk, dict(cu_q=cu[:2])),
                      (chunk, dict(first=f.float())), (chunk, dict(slots=_i32([0] * 5), cu_q=_i32([0] * 6))), (chunk, dict(q=q.cpu())),
                      (chunk, dict(q=torch.zeros((2, 4, 128), dtype=torch.bfloat16, device=DEV)[:, :, :64])),
                      (fill, dict(first=None)), (fill, dict(k=kv.float())), (fill, dict(v=kv[:1])), (fill, dict(layer=5)), (fill, dict(sm_scale=0.0))):
        with pytest.raises(B.BreadcrumbsError) as e:
            call(**bad)
        assert e.value.status == B.BC_ERR_INVALID_ARG
    lib, p = B.lib(), q.data_ptr()
    assert lib.bc_chunk_attn(cache.handle, 0, sl.data_ptr(), None, cu.data_ptr(), 2, 2, p + 8, out.data_ptr(), 1.0, None) == B.BC_ERR_INVALID_ARG
    assert lib.bc_chunk_attn(cache.handle, 0, sl.data_ptr(), None, cu.data_ptr(), 2, (1 << 28) + 1, p, out.data_ptr(), 1.0, None) == B.BC_ERR_UNSUPPORTED
    assert lib.bc_chunk_attn(cache.handle, 0, sl.data_ptr(), None, cu.data_ptr(), 2, 0, None, None, 1.0, None) == B.BC_OK       # nothing to do
    torch.cuda.synchronize()
    assert float(out.min()) == 7.0
    chunk()                                                    # closed slots: zeros
    assert float(out.abs().max()) == 0.0


def test_prompt_chunks_steps_and_sampling_together():
    """The operators as a generation uses them, one layer: prompts processed in chunks from packed projections (norm, rotation, store,
    attention), decode steps from packed projections, every next token sampled from the outputs, compression when a window is full."""
    Hkv, G, D, c, theta, eps = 2, 3, 64, 4, 1e4, 1e-6
    Hq, scale, n = Hkv * G, 1 / 8.0, 3
    width, vocab = (Hq + 2 * Hkv) * D, 501
    plens = [57, 8, 33]
    pair = Pair(1, Hkv, Hq, D, 16, max_seqs=n, num_pages=60, max_pages_per_seq=20, c_default=c)
    slots = list(range(n))
    pair.open(slots, plens)
    g = _gen(18)
    emb, head = randn_bf16(g, (vocab, width), DEV), randn_bf16(g, (Hq * D, vocab), DEV, scale=0.3)
    wq, wk = randn_bf16(g, (D,), DEV), randn_bf16(g, (D,), DEV)
    seqs = [SeqCache(1, c) for _ in range(n)]
    K, V = [np.zeros((0, Hkv, D)) for _ in range(n)], [np.zeros((0, Hkv, D)) for _ in range(n)]
    sl, last = _i32(slots), [None] * n
    for at in range(0, max(plens), 20):
        ms = [max(0, min(20, p - at)) for p in plens]
        first = [min(at, p) for p in plens]
        total = sum(ms)
        pos = torch.cat([torch.arange(f, f + m) for f, m in zip(first, ms)]).to(DEV, torch.int32)
        qkv = emb[torch.randint(0, vocab, (total,), generator=g, device=DEV)]
        q, k, v = B.bc_norm_rope_split(qkv, pos, theta, wq, wk, eps, Hq, Hkv)
        rq, rk, _ = norm_rope_split(f64(qkv), f64(pos), Hq, Hkv, D, theta, f64(wq), f64(wk), eps)
        assert np.abs(f64(q) - rq).max() <= 2.0 ** -8 * np.abs(rq).max() + 1e-4 and np.abs(f64(k) - rk).max() <= 2.0 ** -8 * np.abs(rk).max() + 1e-4
        out = torch.empty((total, Hq, D), dtype=torch.bfloat16, device=DEV)
        pair.gpu.bc_prefill_chunk(0, sl, _i32(first), _cu(ms), total, q, k, v, out, scale)
        a = 0
        for i, m in enumerate(ms):
            K[i], V[i] = np.concatenate([K[i], f64(k)[a:a + m]]), np.concatenate([V[i], f64(v)[a:a + m]])
            r, mag = chunk_attend(f64(q)[a:a + m], K[i], V[i], first[i], scale)
            _assert_chunk(out[a:a + m], r, mag)
            if m and first[i] + m == plens[i]:
                last[i] = out[a + m - 1]
            a += m
    for i in range(n):
        seqs[i].prefill(0, K[i], V[i])
    par = dict(temperature=torch.tensor([0.8, 1.0, 0.0], device=DEV), top_k=_i32([40, 0, 0]), top_p=torch.tensor([0.9, 0.8, 1.0], device=DEV),
               min_p=torch.tensor([0.0, 0.05, 0.0], device=DEV))
    x, pos = torch.stack(last), _i32(plens)
    for t in range(1, 2 * c + 2):
        logits, u = x.reshape(n, -1) @ head, torch.rand(n, generator=g, device=DEV)
        tok = B.bc_sample(logits, u, **par)
        assert tok.tolist() == [sample(f64(logits)[i], float(u[i]), *[float(par[k][i]) if k != "top_k" else int(par[k][i])
                                                                      for k in ("temperature", "top_k", "top_p", "min_p")]) for i in range(n)]
        qkv, x = emb[tok], pair.gpu.new_out(n)
        pair.gpu.bc_norm_rope_decode_step(0, sl, qkv, pos, theta, wq, wk, eps, x, scale)
        q, k, v = B.bc_norm_rope_split(qkv, pos, theta, wq, wk, eps, Hq, Hkv)
        for i in range(n):
            seqs[i].append(0, f64(k)[i], f64(v)[i])
            ref, mag = chunk_attend(f64(q)[i:i + 1], *seqs[i].entries(0), 1 << 20, scale)
            _assert_chunk(x[i:i + 1], ref, mag)
        pos = pos + 1
        if t % c == 0:
            bk, bv = randn_bf16(g, (n, Hkv, D), DEV), randn_bf16(g, (n, Hkv, D), DEV)
            pair.gpu.bc_compress(0, sl, bk, bv)
            for i in range(n):
                seqs[i].compress(0, f64(bk)[i], f64(bv)[i])
            pos = pos + 1
    w = [1] * n                                                # the window's tokens again, at once
    chunk = torch.empty((n, Hq, D), dtype=torch.bfloat16, device=DEV)
    pair.gpu.bc_chunk_attn(0, sl, _cu(w), n, q, chunk, scale)
    for i in range(n):
        _assert_chunk(chunk[i:i + 1], *chunk_attend(f64(q)[i:i + 1], *seqs[i].entries(0), 1 << 20, scale))
    assert pair.gpu.bc_poll_error()[0] == 0
