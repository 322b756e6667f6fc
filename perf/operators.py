"""Cases and plain forms of the operators around the compressed cache: attention of a chunk of new tokens over the
paged cache, norm and rotation of query and key heads (forward and gradient), and sampling of the next token.

run(state) computes an operator in its plain form (elementary torch operations), or, where `own` is true, by the
library's calls.  exact(case, seed) is the operator's definition in 64 bits, written apart from both.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6


def listed():
    return [
        # a short follow-up turn on a stored prompt of one conversation: the smallest call, latency counts
        dict(name="chunk_turn", op="chunk", n=1, q_lo=13, q_hi=13, hist_lo=499, hist_hi=499, c=1, gen=0, q_heads=12,
             kv_heads=2, head_dim=128, page=16, store=True),
        # the sweep's batch (64 sequences, 32 / 8 heads, ratio 16): five guessed tokens of each are checked at once
        dict(name="chunk_check", op="chunk", n=64, q_lo=5, q_hi=5, hist_lo=256, hist_hi=768, c=16, gen=1033, q_heads=32,
             kv_heads=8, head_dim=128, page=16, store=False),
        # single tokens over long uncompressed caches: few rows, one long axis
        dict(name="chunk_single_long", op="chunk", n=3, q_lo=1, q_hi=1, hist_lo=30011, hist_hi=32000, c=1, gen=200,
             q_heads=12, kv_heads=2, head_dim=128, page=16, store=False),
        # a ragged mix of prompt chunks and single tokens, 64-wide heads, pages that divide no tile
        dict(name="chunk_ragged", op="chunk", n=33, q_lo=1, q_hi=257, hist_lo=0, hist_hi=4000, c=1, gen=0, q_heads=14,
             kv_heads=2, head_dim=64, page=24, store=True),
        # chunked prompt processing at full rate: 4 x 2048 new tokens behind 6144 stored ones
        dict(name="chunk_prefill", op="chunk", n=4, q_lo=2048, q_hi=2048, hist_lo=6144, hist_hi=6144, c=1, gen=0,
             q_heads=32, kv_heads=8, head_dim=128, page=16, store=True),
        # one decode step of the 1.5B shape at batch 64: a launch's latency
        dict(name="rope_decode", op="rope", n=64, q_heads=12, kv_heads=2, head_dim=128, theta=1e6, pad=0, far=40000),
        # a prompt chunk of the sweep's head counts: bandwidth
        dict(name="rope_prefill", op="rope", n=16384, q_heads=32, kv_heads=8, head_dim=128, theta=1e6, pad=0, far=131072),
        # odd row count, 64-wide heads, rows inside a wider fused projection
        dict(name="rope_odd", op="rope", n=4099, q_heads=14, kv_heads=1, head_dim=64, theta=1e4, pad=24, far=9000),
        # the gradient for a batch of teacher-forced trajectories
        dict(name="rope_grad", op="rope_grad", n=8192, q_heads=32, kv_heads=8, head_dim=128, theta=1e6, pad=0, far=32768),
        # the same for one short trajectory of the 1.5B shape
        dict(name="rope_grad_short", op="rope_grad", n=257, q_heads=12, kv_heads=2, head_dim=128, theta=1e6, pad=8, far=2000),
        # the decoding step of a batch of 64 on the 1.5B shape's vocabulary, nucleus sampling
        dict(name="sample_batch", op="sample", n=64, vocab=151936, pad=0, f32=False, temperature=0.7, top_k=0, top_p=0.95,
             min_p=0.0),
        # a few rows, 32-bit logits of an odd vocabulary inside a padded row, all filters at once
        dict(name="sample_few", op="sample", n=3, vocab=50257, pad=47, f32=True, temperature=1.0, top_k=50, top_p=0.9,
             min_p=0.02),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["chunk", "chunk", "rope", "rope_grad", "sample"])
    heads = rng.choice([(12, 2), (32, 8), (14, 2), (8, 2), (4, 4), (16, 1), (28, 4)])
    if kind == "chunk":
        d = 128 if rng.random() < 0.6 else 64
        page = rng.choice([16, 16, 16, 64, 24, 8, 1, 7])
        store = rng.random() < 0.6
        n = _log_int(rng, 1, 48)
        top = max(1, min(2048, 8192 // n))
        hist = max(1, min(_log_int(rng, 1, 12000), 200000 // n))
        if store:
            q_hi = _log_int(rng, 1, top)
            c, gen = 1, 0
        else:
            c = rng.choice([1, 4, 16, 32])
            gen = _log_int(rng, 8, 3000) if c > 1 else _log_int(rng, 8, 1000)
            live = gen if c == 1 else gen % c
            if live == 0:
                gen, live = gen + 3, 3
            q_hi = min(live, _log_int(rng, 1, 64))
        return dict(op="chunk", n=n, q_lo=max(1, q_hi // 3), q_hi=q_hi, hist_lo=hist // 4, hist_hi=hist, c=c, gen=gen,
                    q_heads=heads[0], kv_heads=heads[1], head_dim=d, page=page, store=store)
    if kind in ("rope", "rope_grad"):
        d = rng.choice([64, 128])
        return dict(op=kind, n=_log_int(rng, 1, 8000), q_heads=heads[0], kv_heads=heads[1], head_dim=d,
                    theta=rng.choice([1e4, 5e5, 1e6]), pad=rng.choice([0, 0, 8, 64]), far=_log_int(rng, 16, 200000))
    return dict(op="sample", n=_log_int(rng, 1, 64), vocab=_log_int(rng, 2, 150000), pad=rng.choice([0, 0, 1, 8]),
                f32=rng.random() < 0.3, temperature=rng.choice([0.3, 0.6, 0.8, 1.0, 1.5]),
                top_k=rng.choice([0, 0, 1, 20, 50, 400]), top_p=rng.choice([1.0, 0.5, 0.8, 0.95, 0.99]),
                min_p=rng.choice([0.0, 0.0, 0.05, 0.3]))


# ---- inputs ------------------------------------------------------------------------------------------------------
def _spread(n, lo, hi):
    """n lengths between lo and hi, unordered, the same for every seed."""
    return [hi if n == 1 else lo + int(((i * 0.6180339887 + 0.5) % 1.0) * (hi - lo + 1)) for i in range(n)]


def _lengths(case):
    """Per sequence: queries, prompt entries, beacons, window entries, logical index of the first query."""
    qs = _spread(case["n"], case["q_lo"], case["q_hi"])
    hist = _spread(case["n"], case["hist_lo"], case["hist_hi"])
    gen, c = case["gen"], case["c"]
    nb = gen // c if c > 1 else 0
    w = gen % c if c > 1 else gen
    if case["store"]:
        return [(q, h + q, 0, 0, h) for q, h in zip(qs, hist)]
    return [(q, h, nb, w, h + nb + w - q) for q, h in zip(qs, hist)]


def _i32(xs):
    return torch.tensor(list(xs), dtype=torch.int32, device=DEV)


def _cu(xs):
    return _i32(np.concatenate([[0], np.cumsum(xs)]))


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rnd = lambda *s, scale=1.0: (torch.randn(s, generator=g, device=DEV) * scale).to(torch.bfloat16)
    s = dict(case=case)
    if case["op"] == "chunk":
        n, ps, hq, hk, d = case["n"], case["page"], case["q_heads"], case["kv_heads"], case["head_dim"]
        lens = _lengths(case)
        s.update(total_q=sum(x[0] for x in lens), max_q=max(x[0] for x in lens), max_len=max(x[1] + x[2] + x[3] for x in lens),
                 cu_q=_cu([x[0] for x in lens]), first=_i32(x[4] for x in lens), prompt=_i32(x[1] for x in lens),
                 beacons=_i32(x[2] for x in lens), window=_i32(x[3] for x in lens), scale=1.0 / math.sqrt(d),
                 slots=_i32(range(n)))
        s["q"] = rnd(s["total_q"], hq, d)
        # what the sequences hold already, packed: stored prompt entries, then beacons, then the window's entries
        stored = [x[4] if case["store"] else x[1] for x in lens]
        s.update(stored=sum(stored), cu_stored=_cu(stored), hist_k=rnd(sum(stored), hk, d), hist_v=rnd(sum(stored), hk, d))
        nb, w = lens[0][2], lens[0][3]
        s.update(bea_k=rnd(n * nb, hk, d), bea_v=rnd(n * nb, hk, d), win_k=rnd(n * w, hk, d), win_v=rnd(n * w, hk, d))
        if case["store"]:
            s.update(k=rnd(s["total_q"], hk, d), v=rnd(s["total_q"], hk, d))
        # the plain form's paged store: pages in an arbitrary order, a table of prompt, beacon and window pages
        cols = [max(-(-x[j] // ps) for x in lens) for j in (1, 2, 3)]
        per = sum(cols)
        s["cols"] = cols
        s["table"] = torch.randperm(n * per, generator=g, device=DEV).view(n, per)
        s["pool_k"] = torch.zeros((n * per * ps, hk, d), dtype=torch.bfloat16, device=DEV)
        s["pool_v"] = torch.zeros_like(s["pool_k"])
        seq = torch.repeat_interleave(torch.arange(n, device=DEV), torch.tensor(stored, device=DEV))
        pos = torch.arange(s["stored"], device=DEV) - s["cu_stored"].long()[seq]
        _put(s, seq, pos, s["hist_k"], s["hist_v"])
        off = s["prompt"].long()
        for cnt, k, v in ((nb, s["bea_k"], s["bea_v"]), (w, s["win_k"], s["win_v"])):
            seq = torch.arange(n, device=DEV).repeat_interleave(cnt)
            _put(s, seq, off[seq] + torch.arange(cnt, device=DEV).repeat(n), k, v)
            off = off + cnt
        if own:  # the cache that a serving program keeps: opened, and holding what the sequences hold before the call
            s["cache"] = _cache(s)
            s["out"] = torch.empty_like(s["q"])
    elif case["op"] in ("rope", "rope_grad"):
        n, hq, hk, d = case["n"], case["q_heads"], case["kv_heads"], case["head_dim"]
        width = (hq + 2 * hk) * d
        s["qkv"] = rnd(n, width + case["pad"])[:, :width]
        s["positions"] = torch.randint(0, case["far"], (n,), generator=g, device=DEV, dtype=torch.int32)
        s["q_weight"], s["k_weight"] = 1 + rnd(d, scale=0.2), 1 + rnd(d, scale=0.2)
        if case["op"] == "rope_grad":
            s.update(dq=rnd(n, hq, d), dk=rnd(n, hk, d), dv=rnd(n, hk, d))
    else:
        n, v = case["n"], case["vocab"]
        x = torch.randn((n, v + case["pad"]), generator=g, device=DEV) * 2.2
        # a handful of likely tokens above a broad rest, a few tokens ruled out
        x[:, :v].scatter_add_(1, torch.randint(0, v, (n, 24), generator=g, device=DEV), 4 + 3 * torch.randn((n, 24), generator=g, device=DEV))
        x[:, :v].scatter_(1, torch.randint(0, v, (n, 3), generator=g, device=DEV), -math.inf)
        x[:, 0] = 0.5
        s["logits"] = (x if case["f32"] else x.to(torch.bfloat16))[:, :v]
        rows = torch.arange(n, device=DEV)
        t = torch.full((n,), case["temperature"], device=DEV)
        s["temperature"] = torch.where(rows % 8 == 7, torch.zeros_like(t), t * (1 + 0.05 * (rows % 3)))
        s["top_k"] = torch.full((n,), case["top_k"], dtype=torch.int32, device=DEV)
        s["top_p"] = torch.full((n,), case["top_p"], device=DEV)
        s["min_p"] = torch.full((n,), case["min_p"], device=DEV)
        s["uniform"] = torch.rand((n,), generator=g, device=DEV)
    return s


def _cache(s):
    from paper_2510_13797_b200 import binding as B
    c = s["case"]
    n, ps, hk, d = c["n"], c["page"], c["kv_heads"], c["head_dim"]
    lens = _lengths(c)
    pages = [-(-x[1] // ps) + -(-x[2] // ps) + -(-x[3] // ps) + 1 for x in lens]
    cache = B.Cache(1, hk, c["q_heads"], d, c["c"], ps, n, sum(pages), max(pages))
    cache.bc_seq_open(s["slots"], s["prompt"])
    cache.bc_prefill(0, s["slots"], s["cu_stored"], s["stored"], s["hist_k"], s["hist_v"])
    if c["gen"]:  # the generated tokens that compression has evicted are never read: only the window's rows count
        w = lens[0][3]
        tok = lambda win: torch.cat([torch.zeros((n, c["gen"] - w, hk, d), dtype=torch.bfloat16, device=DEV), win.view(n, w, hk, d)], 1)
        cache.bc_restore(0, s["slots"], _cu([c["gen"]] * n), n * c["gen"], n * lens[0][2], tok(s["win_k"]).contiguous(),
                         tok(s["win_v"]).contiguous(), s["bea_k"], s["bea_v"])
    return cache


# ---- chunk attention, plain ---------------------------------------------------------------------------------------
def _rows(s, seq, entry):
    """Rows of the plain form's store that hold the logical entries `entry` of sequences `seq`."""
    ps, (c0, c1, _) = s["case"]["page"], s["cols"]
    p, b = s["prompt"].long()[seq], s["beacons"].long()[seq]
    in_p, in_b = entry < p, entry < p + b
    pos = torch.where(in_p, entry, torch.where(in_b, entry - p, entry - p - b))
    col = torch.where(in_p, 0, torch.where(in_b, c0, c0 + c1)) + pos // ps
    return s["table"][seq, col.clamp(0, s["table"].shape[1] - 1)] * ps + pos % ps


def _put(s, seq, entry, k, v):
    rows = _rows(s, seq, entry)
    s["pool_k"][rows], s["pool_v"][rows] = k, v


def _chunk_plain(s):
    c = s["case"]
    n, hq, hk, d, mq = c["n"], c["q_heads"], c["kv_heads"], c["head_dim"], s["max_q"]
    cu, total = s["cu_q"].long(), s["total_q"]
    seq = torch.repeat_interleave(torch.arange(n, device=DEV), cu[1:] - cu[:-1], output_size=total)
    r = torch.arange(total, device=DEV) - cu[seq]
    if c["store"]:
        _put(s, seq, s["first"].long()[seq] + r, s["k"], s["v"])
    entry = torch.arange(s["max_len"], device=DEV).expand(n, -1)
    live = (s["prompt"] + s["beacons"] + s["window"]).long()
    rows = _rows(s, torch.arange(n, device=DEV)[:, None], torch.minimum(entry, (live - 1).clamp(min=0)[:, None]))
    k = s["pool_k"][rows].float().permute(0, 2, 3, 1)                                # [n, hk, d, len]
    v = s["pool_v"][rows].float().transpose(1, 2)                                    # [n, hk, len, d]
    q = torch.zeros((n, mq, hk, hq // hk, d), device=DEV)
    q[seq, r] = s["q"].float().view(total, hk, hq // hk, d)
    q = q.permute(0, 2, 3, 1, 4).reshape(n, hk, (hq // hk) * mq, d)
    w = torch.matmul(q, k).mul_(s["scale"]).view(n, hk, hq // hk, mq, -1)
    vis = torch.minimum(s["first"].long()[:, None] + torch.arange(mq, device=DEV) + 1, live[:, None])
    w.masked_fill_((entry[:, None, :] >= vis[:, :, None])[:, None, None], -math.inf)
    top = w.amax(-1, keepdim=True)
    w.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total_w = w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(n, hk, -1, w.shape[-1]), v).view(n, hk, hq // hk, mq, d)
    o = torch.where(total_w > 0, o / total_w, torch.zeros_like(o))
    return o.permute(0, 3, 1, 2, 4).reshape(n, mq, hq, d)[seq, r].to(torch.bfloat16)


# ---- norm and rotation, plain -------------------------------------------------------------------------------------
def _angles(s):
    d = s["case"]["head_dim"]
    freq = s["case"]["theta"] ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=DEV) / d)
    a = s["positions"].double()[:, None] * freq
    return a.cos().float()[:, None], a.sin().float()[:, None]


def _heads(s):
    c = s["case"]
    n, hq, hk, d = c["n"], c["q_heads"], c["kv_heads"], c["head_dim"]
    x = s["qkv"].reshape(n, hq + 2 * hk, d)
    return x[:, :hq].float(), x[:, hq:hq + hk].float(), x[:, hq + hk:]


def _norm_rope(x, w, cos, sin):
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    lo, hi = y.chunk(2, -1)
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1).to(torch.bfloat16)


def _norm_rope_grad(x, w, cos, sin, g):
    lo, hi = g.float().chunk(2, -1)
    dy = torch.cat([lo * cos + hi * sin, hi * cos - lo * sin], -1)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    dw = (x * r * dy).double().sum((0, 1)).float()
    gw = dy * w.float()
    return (r * (gw - x * (r * r * (x * gw).mean(-1, keepdim=True)))).to(torch.bfloat16), dw


# ---- sampling, plain ----------------------------------------------------------------------------------------------
def _sample_plain(s):
    x = s["logits"].double()
    n, v = x.shape
    x = torch.where(x.isnan(), torch.full_like(x, -math.inf), x)
    best = x.amax(-1, keepdim=True)
    at = torch.arange(v, device=DEV)
    greedy = torch.where(x == best, at, v).amin(-1)
    t = s["temperature"].double()[:, None]
    e = torch.where(x == -math.inf, torch.zeros_like(x), ((x - best) / torch.where(t > 0, t, torch.ones_like(t))).exp())
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    es = e.gather(1, order)
    k = s["top_k"].long()[:, None]
    es = torch.where((k <= 0) | (at < k), es, torch.zeros_like(es))
    p = s["top_p"].double()[:, None]
    before = es.cumsum(-1).roll(1, -1)
    before[:, 0] = 0
    keep = (es > 0) & ((p >= 1) | (at == 0) | (before < p * es.sum(-1, keepdim=True)))
    kept = torch.zeros_like(keep).scatter_(1, order, keep) & (e >= s["min_p"].double()[:, None])
    cum = torch.where(kept, e, torch.zeros_like(e)).cumsum(-1)
    j = (cum <= s["uniform"].double()[:, None] * cum[:, -1:]).sum(-1)
    last = torch.where(kept, at, -1).amax(-1)
    return torch.where(t[:, 0] > 0, torch.minimum(j, last), greedy)


def run(s):
    c = s["case"]
    if own:
        from paper_2510_13797_b200 import binding as B
        if c["op"] == "chunk" and c["store"]:
            s["cache"].bc_prefill_chunk(0, s["slots"], s["first"], s["cu_q"], s["total_q"], s["q"], s["k"], s["v"], s["out"], s["scale"])
            return s["out"]
        if c["op"] == "chunk":
            s["cache"].bc_chunk_attn(0, s["slots"], s["cu_q"], s["total_q"], s["q"], s["out"], s["scale"])
            return s["out"]
        if c["op"] == "rope":
            return B.bc_norm_rope_split(s["qkv"], s["positions"], c["theta"], s["q_weight"], s["k_weight"], EPS, c["q_heads"], c["kv_heads"])
        if c["op"] == "rope_grad":
            return B.bc_norm_rope_split_backward(s["qkv"], s["positions"], c["theta"], s["q_weight"], s["k_weight"], EPS, s["dq"],
                                                 s["dk"], s["dv"])
        return B.bc_sample(s["logits"], s["uniform"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
    if c["op"] == "chunk":
        return _chunk_plain(s)
    if c["op"] == "sample":
        return _sample_plain(s)
    q, k, v = _heads(s)
    cos, sin = _angles(s)
    if c["op"] == "rope":
        return _norm_rope(q, s["q_weight"], cos, sin), _norm_rope(k, s["k_weight"], cos, sin), v.contiguous()
    gq, wq = _norm_rope_grad(q, s["q_weight"], cos, sin, s["dq"])
    gk, wk = _norm_rope_grad(k, s["k_weight"], cos, sin, s["dk"])
    return torch.cat([gq, gk, s["dv"]], 1).view(c["n"], -1), wq, wk


def work(case):
    d = case.get("head_dim", 0)
    if case["op"] == "chunk":
        lens = _lengths(case)
        hq, hk = case["q_heads"], case["kv_heads"]
        rows = sum(x[0] for x in lens)
        seen = sum(x[4] + x[0] for x in lens)                                        # entries some query sees
        pairs = sum(x[0] * (x[4] + 1) + x[0] * (x[0] - 1) // 2 for x in lens)
        fresh = rows if case["store"] else 0                                         # read from the inputs, written to the cache
        return dict(bytes=4 * rows * hq * d + 4 * hk * d * (seen + fresh), flops=4 * d * hq * pairs)
    if case["op"] in ("rope", "rope_grad"):
        n, hq, hk = case["n"], case["q_heads"], case["kv_heads"]
        rot, every = n * (hq + hk) * d, n * (hq + 2 * hk) * d
        if case["op"] == "rope":
            return dict(bytes=4 * every + 4 * n + 4 * d, flops=10 * rot)
        return dict(bytes=2 * rot + 4 * every + 4 * n + 12 * d, flops=20 * rot)
    n, v = case["n"], case["vocab"]
    return dict(bytes=n * v * (4 if case["f32"] else 2) + 28 * n, flops=6 * n * v)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "chunk":
        hq, hk, d, n = case["q_heads"], case["kv_heads"], case["head_dim"], case["n"]
        out = torch.zeros((s["total_q"], hq, d), dtype=torch.float64, device=DEV)
        lens, a, h0 = _lengths(case), 0, 0
        for i, (m, p, nb, w, first) in enumerate(lens):
            stored = first if case["store"] else p
            parts = lambda h, b, wi, new: torch.cat([h[h0:h0 + stored], b[i * nb:(i + 1) * nb], wi[i * w:(i + 1) * w]]
                                                    + ([new[a:a + m]] if case["store"] else [])).double()
            k, v = parts(s["hist_k"], s["bea_k"], s["win_k"], s.get("k")), parts(s["hist_v"], s["bea_v"], s["win_v"], s.get("v"))
            hidden = torch.arange(k.shape[0], device=DEV)[None, :] > torch.arange(first, first + m, device=DEV)[:, None]
            for h in range(hq):
                z = (s["q"][a:a + m, h].double() @ k[:, h * hk // hq].T) / math.sqrt(d)
                out[a:a + m, h] = torch.softmax(z.masked_fill(hidden, -math.inf), -1) @ v[:, h * hk // hq]
            a, h0 = a + m, h0 + stored
        return out
    if case["op"] in ("rope", "rope_grad"):
        hq, hk, d = case["q_heads"], case["kv_heads"], case["head_dim"]
        x = s["qkv"].double().reshape(case["n"], -1, d)
        j = torch.arange(d // 2, dtype=torch.float64, device=DEV)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s["positions"].double()[:, None, None] * torch.pow(
            torch.tensor(case["theta"], dtype=torch.float64, device=DEV), -2 * j / d))
        pair = lambda y: torch.complex(y[..., :d // 2].contiguous(), y[..., d // 2:].contiguous())
        flat = lambda z: torch.cat([z.real, z.imag], -1)
        unit = lambda y: y / torch.sqrt((y ** 2).sum(-1, keepdim=True) / d + EPS)
        xs = (x[:, :hq], x[:, hq:hq + hk])
        ws = (s["q_weight"].double(), s["k_weight"].double())
        if case["op"] == "rope":
            return tuple(flat(pair(unit(y) * w) * turn) for y, w in zip(xs, ws)) + (x[:, hq + hk:],)
        grads, dws = [], []
        for y, w, g in zip(xs, ws, (s["dq"], s["dk"])):
            back = flat(pair(g.double()) * turn.conj())
            norm = torch.sqrt((y ** 2).sum(-1, keepdim=True) / d + EPS)
            dws.append((unit(y) * back).sum((0, 1)))
            grads.append(w * back / norm - y * ((w * back * y).sum(-1, keepdim=True) / (d * norm ** 3)))
        return torch.cat(grads + [s["dv"].double()], 1).view(case["n"], -1), dws[0], dws[1]
    x = s["logits"].double().cpu().numpy()
    par = {k: s[k].cpu().numpy() for k in ("temperature", "top_k", "top_p", "min_p", "uniform")}
    out = []
    for r in range(case["n"]):
        t, k, p = float(par["temperature"][r]), int(par["top_k"][r]), float(par["top_p"][r])
        if t <= 0:
            out.append(int(np.flatnonzero(x[r] == x[r].max())[0]))
            continue
        order = np.lexsort((np.arange(x.shape[1]), -x[r]))
        e = np.exp((x[r] - x[r].max()) / t)
        if k > 0:
            order = order[:k]
        if p < 1:
            c = np.cumsum(e[order])
            order = order[:1 + int(np.searchsorted(c, p * c[-1], side="left"))]
        chosen = np.sort(order[e[order] >= float(par["min_p"][r])])
        c = np.cumsum(e[chosen])
        out.append(int(chosen[min(int(np.searchsorted(c, float(par["uniform"][r]) * c[-1], side="right")), len(chosen) - 1)]))
    return torch.tensor(out, dtype=torch.int64)
