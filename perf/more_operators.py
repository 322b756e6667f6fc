"""Cases and plain forms of the operators that training a student on compressed trajectories needs beside the mask form and
the distillation loss: log-probabilities of given tokens with entropy and the most likely alternatives (forward and gradient),
the norms around a block with its gate and residual scale (forward and gradient), and the gradient of the mask form.

run(state) computes an operator in its plain form (elementary torch operations), or, where `own` is true, by the
library's calls.  exact(case, seed) is the operator's definition in 64 bits, written apart from both.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
NONE = -100        # the target of a position that is not trained on


def listed():
    return [
        # one conversation's decoding step that reports its token's log-probability and five alternatives: latency counts
        dict(name="logp_one", op="logp", n=1, vocab=50257, pad=47, f32=True, top_k=5),
        # the decoding step of a batch of 64 on the 1.5B shape's vocabulary, with twenty alternatives
        dict(name="logp_batch", op="logp", n=64, vocab=151936, pad=0, f32=False, top_k=20),
        # a teacher's pass over trajectories: the hundred likeliest tokens of every position, as the distillation loss takes them
        dict(name="logp_teacher", op="logp", n=2048, vocab=151936, pad=0, f32=False, top_k=100),
        # the gradient of a policy objective with an entropy term over those positions
        dict(name="logp_grad", op="logp_grad", n=2048, vocab=151936, pad=0, f32=False, top_k=0),
        # the same for a few positions with 32-bit logits in padded rows of an odd vocabulary
        dict(name="logp_grad_odd", op="logp_grad", n=37, vocab=50257, pad=3, f32=True, top_k=0),
        # one decode step of the 1.5B shape at batch 64: a launch's latency
        dict(name="norm_decode", op="norm", n=64, hidden=1536, gate="none", post=True, scale=1.0),
        # a prompt chunk of the sweep's width, a gate value for every element: bandwidth
        dict(name="norm_prefill", op="norm", n=16384, hidden=4096, gate="rows", post=True, scale=0.5),
        # the gradient for a batch of trajectories, one gate vector for all rows
        dict(name="norm_grad", op="norm_grad", n=8192, hidden=4096, gate="vector", post=True, scale=0.5),
        # the same for one short trajectory of the 1.5B shape without the norm behind the block, a gate value for every element
        dict(name="norm_grad_short", op="norm_grad", n=257, hidden=1536, gate="rows", post=False, scale=1.0),
        # the mask form's gradient for one short trajectory of the 1.5B shape
        dict(name="mask_grad_short", op="mask_grad", n=1, p_lo=71, p_hi=71, t_lo=509, t_hi=509, c=16, q_heads=12, kv_heads=2),
        # a ragged batch, a group of 7 heads, many beacons
        dict(name="mask_grad_ragged", op="mask_grad", n=5, p_lo=0, p_hi=900, t_lo=130, t_hi=2050, c=2, q_heads=14, kv_heads=2),
        # trajectories of the sweep's shape at its middle ratio: tensor-core rate
        dict(name="mask_grad_batch", op="mask_grad", n=4, p_lo=512, p_hi=512, t_lo=6000, t_hi=6000, c=16, q_heads=32, kv_heads=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logp", "logp_grad", "norm", "norm_grad", "mask_grad", "mask_grad"])
    if op in ("logp", "logp_grad"):
        vocab = _log_int(rng, 2, 151936)
        return dict(op=op, n=_log_int(rng, 1, 1000), vocab=vocab, pad=rng.choice([0, 0, 1, 8]), f32=rng.random() < 0.3,
                    top_k=min(vocab, rng.choice([0, 1, 5, 20, 64, 100, 128])) if op == "logp" else 0)
    if op in ("norm", "norm_grad"):
        return dict(op=op, n=_log_int(rng, 1, 6000), hidden=8 * _log_int(rng, 1, 512), gate=rng.choice(["none", "vector", "rows"]),
                    post=rng.random() < 0.6, scale=rng.choice([1.0, 0.5, 0.22]))
    heads = rng.choice([(12, 2), (32, 8), (14, 2), (8, 2), (4, 4), (16, 1), (24, 8)])
    n = _log_int(rng, 1, 6)
    t_hi = min(7000 // n, _log_int(rng, 1, 3500))
    p_hi = rng.choice([0, _log_int(rng, 1, 500)])
    return dict(op=op, n=n, p_lo=p_hi // 4, p_hi=p_hi, t_lo=max(1, t_hi // 3), t_hi=t_hi, c=rng.choice([1, 2, 4, 8, 16, 32, 50]),
                q_heads=heads[0], kv_heads=heads[1])


# ---- inputs ------------------------------------------------------------------------------------------------------
def _spread(n, lo, hi):
    """n lengths between lo and hi, unordered, the same for every seed."""
    return [hi if n == 1 else lo + int(((i * 0.6180339887 + 0.5) % 1.0) * (hi - lo + 1)) for i in range(n)]


def _lengths(case):
    """Prompt entries, generated tokens and beacons of every trajectory."""
    p, t = _spread(case["n"], case["p_lo"], case["p_hi"]), _spread(case["n"], case["t_lo"], case["t_hi"])
    return p, t, [x // case["c"] if case["c"] > 1 else 0 for x in t]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rnd = lambda *s, scale=1.0: (torch.randn(s, generator=g, device=DEV) * scale).to(torch.bfloat16)
    s = dict(case=case)
    n = case["n"]
    if case["op"] in ("logp", "logp_grad"):
        v = case["vocab"]
        x = torch.randn((n, v + case["pad"]), generator=g, device=DEV) * 2.2
        # a handful of likely tokens above a broad rest, a few tokens ruled out
        x[:, :v].scatter_add_(1, torch.randint(0, v, (n, 24), generator=g, device=DEV), 4 + 3 * torch.randn((n, 24), generator=g, device=DEV))
        x[:, :v].scatter_(1, torch.randint(0, v, (n, 3), generator=g, device=DEV), -math.inf)
        x[:, 0] = 0.5
        s["logits"] = (x if case["f32"] else x.to(torch.bfloat16))[:, :v]
        # the tokens were sampled: mostly likely ones, never a ruled-out one; some positions are not trained on
        u = torch.rand((n, 8), generator=g, device=DEV)
        picks = (u * v).long().clamp(max=v - 1)
        z = s["logits"].gather(1, picks).float()
        best = picks.gather(1, z.argmax(1, keepdim=True))[:, 0]
        best = torch.where(s["logits"].gather(1, best[:, None])[:, 0] == -math.inf, torch.zeros_like(best), best)
        skip = torch.rand((n,), generator=g, device=DEV) < 0.06
        s["targets"] = torch.where(skip, torch.full_like(best, NONE), best)
        if case["op"] == "logp_grad":
            s["stats"], s["entropy"] = _moments(s["logits"].float())
            s["d_logprob"] = torch.randn((n,), generator=g, device=DEV)
            s["d_entropy"] = 0.1 * torch.randn((n,), generator=g, device=DEV)
    elif case["op"] in ("norm", "norm_grad"):
        h = case["hidden"]
        s.update(x=rnd(n, h, scale=3.0), h=rnd(n, h, scale=2.0), post_weight=1 + rnd(h, scale=0.2) if case["post"] else None,
                 pre_weight=1 + rnd(h, scale=0.2))
        s["gate"] = dict(none=lambda: None, vector=lambda: 1 + rnd(h, scale=0.3), rows=lambda: 1 + rnd(n, h, scale=0.3))[case["gate"]]()
        if case["op"] == "norm_grad":
            s["h"] = _block_norm(s)[0]                                    # what the forward call has left: the new residual stream
            s.update(dh=rnd(n, h), dy=rnd(n, h))
    else:
        p, t, nb = _lengths(case)
        hq, hk, d = case["q_heads"], case["kv_heads"], 128
        s.update(prompt_lens=p, token_lens=t, scale=1.0 / math.sqrt(d), prompt_k=rnd(sum(p), hk, d), prompt_v=rnd(sum(p), hk, d),
                 tok_q=rnd(sum(t), hq, d), tok_k=rnd(sum(t), hk, d), tok_v=rnd(sum(t), hk, d), beacon_q=rnd(sum(nb), hq, d),
                 beacon_k=rnd(sum(nb), hk, d), beacon_v=rnd(sum(nb), hk, d), d_tok=rnd(sum(t), hq, d), d_beacon=rnd(sum(nb), hq, d))
        # what the forward call has left: its outputs and the logarithm of every row's sum
        s.update(zip(("out_tok", "out_beacon", "lse_tok", "lse_beacon"), _mask_forward(s)))
    return s


# ---- log-probabilities, plain -------------------------------------------------------------------------------------
def _moments(x):
    """Per row: its maximum and the logarithm of sum exp(x - maximum); and the entropy of softmax(x)."""
    top = x.amax(-1, keepdim=True)
    y = x - top
    e = y.exp()
    total = e.sum(-1, dtype=torch.float64)
    part = torch.where(e > 0, e * y, torch.zeros_like(e)).sum(-1, dtype=torch.float64)
    log = total.log()
    return torch.stack([top[:, 0], log.float()], 1), (log - part / total).float()


def _logp_plain(s):
    x, t, k = s["logits"].float(), s["targets"], s["case"]["top_k"]
    stats, entropy = _moments(x)
    lp = lambda z: (z - stats[:, :1]) - stats[:, 1:]
    given = lp(x.gather(1, t.clamp(min=0)[:, None]))[:, 0]
    logprob = torch.where(t < 0, torch.zeros_like(given), given)
    if k == 0:
        return logprob, entropy, stats
    z, at = torch.sort(x, dim=-1, descending=True, stable=True)
    return logprob, entropy, stats, at[:, :k].int(), lp(z[:, :k])


def _logp_grad_plain(s):
    x, t = s["logits"].float(), s["targets"]
    lp = (x - s["stats"][:, :1]) - s["stats"][:, 1:]
    p = lp.exp()
    g = torch.where(t < 0, torch.zeros_like(s["d_logprob"]), s["d_logprob"])
    grad = -p * (g[:, None] + s["d_entropy"][:, None] * torch.where(p > 0, lp + s["entropy"][:, None], torch.zeros_like(p)))
    grad.scatter_add_(1, t.clamp(min=0)[:, None], g[:, None])
    return grad.to(s["logits"].dtype)


# ---- norms around a block, plain ----------------------------------------------------------------------------------
def _rms(x):
    return torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)


def _weight(w):
    return 1.0 if w is None else w.float()


def _block_norm(s):
    x, c = s["x"].float(), s["case"]
    u = x * _rms(x) * _weight(s["post_weight"]) if c["post"] else x
    h = (s["h"].float() + c["scale"] * _weight(s["gate"]) * u).to(torch.bfloat16)
    z = h.float()
    return h, (z * _rms(z) * _weight(s["pre_weight"])).to(torch.bfloat16)


def _norm_back(x, w, g):
    """Gradient of x * rms(x) * w for x and for w's elements row by row."""
    r = _rms(x)
    gw = g * _weight(w)
    return r * (gw - x * (r * r * (x * gw).mean(-1, keepdim=True))), g * x * r


def _block_norm_grad(s):
    c, x, h = s["case"], s["x"].float(), s["h"].float()
    total = lambda t: t.sum(0, dtype=torch.float64).float()
    dz, dpre = _norm_back(h, s["pre_weight"], s["dy"].float())
    dh = s["dh"].float() + dz
    u = x * _rms(x) * _weight(s["post_weight"]) if c["post"] else x
    dgate = c["scale"] * dh * u
    du = c["scale"] * _weight(s["gate"]) * dh
    dx, dpost = _norm_back(x, s["post_weight"], du) if c["post"] else (du, None)
    out = [dx.to(torch.bfloat16), dh.to(torch.bfloat16), total(dpre)]
    if c["post"]:
        out.append(total(dpost))
    if c["gate"] != "none":
        out.append(total(dgate) if c["gate"] == "vector" else dgate.to(torch.bfloat16))
    return out


# ---- the mask form, plain: all trajectories padded to one length ----------------------------------------------------
def _pad(parts, lens, places):
    """Packed arrays (rows, heads, d), of each trajectory one after the other, as one padded fp32 array [n, heads, places, d]; and
    where every packed row went."""
    out = torch.zeros((len(lens[0]), parts[0].shape[1], places, parts[0].shape[2]), device=DEV)
    where, base = [], torch.zeros(len(lens[0]), dtype=torch.long, device=DEV)
    for x, ln in zip(parts, (torch.tensor(l, device=DEV) for l in lens)):
        seq = torch.repeat_interleave(torch.arange(ln.numel(), device=DEV), ln)
        row = torch.arange(seq.numel(), device=DEV) - (ln.cumsum(0) - ln)[seq] + base[seq]
        out[seq, :, row] = x.float()
        where.append((seq, row))
        base = base + ln
    return out, where


def _mask_scores(s):
    c = s["case"]
    n, hq, hk, ratio = c["n"], c["q_heads"], c["kv_heads"], c["c"]
    p, t, nb = _lengths(c)
    rows, keys = max(a + b for a, b in zip(t, nb)), max(a + b + e for a, b, e in zip(p, nb, t))
    q, at_q = _pad((s["tok_q"], s["beacon_q"]), (t, nb), rows)
    k, at_k = _pad((s["prompt_k"], s["beacon_k"], s["tok_k"]), (p, nb, t), keys)
    v, _ = _pad((s["prompt_v"], s["beacon_v"], s["tok_v"]), (p, nb, t), keys)
    P, T, N = [torch.tensor(x, device=DEV)[:, None] for x in (p, t, nb)]
    r, j = torch.arange(rows, device=DEV)[None], torch.arange(keys, device=DEV)[None]
    beacon_row = r >= T
    window = torch.where(beacon_row, r - T, r // ratio if ratio > 1 else torch.zeros_like(r))   # the window a row belongs to
    last = torch.where(beacon_row, torch.full_like(window, 1 << 30), r)                         # the last token it may see
    tok = j - P - N                                                                             # a key's token index
    key_window = tok // ratio if ratio > 1 else torch.zeros_like(tok)
    is_b, is_t = ((j >= P) & (tok < 0))[:, None], ((tok >= 0) & (tok < T))[:, None]
    sees_b = (j - P)[:, None] < (window + beacon_row)[:, :, None]
    sees_t = (key_window[:, None] == window[:, :, None]) & (tok[:, None] <= last[:, :, None])
    seen = ((j < P)[:, None] | (is_b & sees_b) | (is_t & sees_t)) & (r < T + N)[:, :, None]     # [n, rows, keys]
    qg = q.view(n, hk, hq // hk, rows, 128)
    w = torch.matmul(qg, k[:, :, None].transpose(-1, -2)).mul_(s["scale"])
    w.masked_fill_(~seen[:, None, None], -math.inf)
    top = w.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    total = w.sub_(top).exp_().sum(-1, keepdim=True)
    w.div_(torch.where(total > 0, total, torch.ones_like(total)))
    return qg, k, v, w, top + total.log(), at_q, at_k


def _mask_forward(s):
    _, _, v, w, lse, at_q, _ = _mask_scores(s)
    o = torch.matmul(w, v[:, :, None]).flatten(1, 2)
    return [o[seq, :, row].to(torch.bfloat16) for seq, row in at_q] + [lse.flatten(1, 2)[seq, :, row, 0] for seq, row in at_q]


def _mask_grad_plain(s):
    qg, k, v, w, _, at_q, at_k = _mask_scores(s)
    _, t, nb = _lengths(s["case"])
    do, _ = _pad((s["d_tok"], s["d_beacon"]), (t, nb), qg.shape[3])
    do = do.view(qg.shape)
    dv = torch.matmul(w.transpose(-1, -2), do).sum(2)
    dw = torch.matmul(do, v[:, :, None].transpose(-1, -2))
    dw.sub_((w * dw).sum(-1, keepdim=True)).mul_(w).mul_(s["scale"])
    dq = torch.matmul(dw, k[:, :, None]).flatten(1, 2)
    dk = torch.matmul(dw.transpose(-1, -2), qg).sum(2)
    take = lambda x, where: [x[seq, :, row].to(torch.bfloat16) for seq, row in where]
    (dpk, dbk, dtk), (dpv, dbv, dtv) = take(dk, at_k), take(dv, at_k)
    dtq, dbq = take(dq, at_q)
    return dpk, dpv, dtq, dtk, dtv, dbq, dbk, dbv


def run(s):
    c = s["case"]
    if own:
        from paper_2510_13797_b200 import binding as B
        if c["op"] == "logp":
            logprob, entropy, stats, top, top_logprob = B.bc_token_logprobs(s["logits"], s["targets"], c["top_k"])
            return (logprob, entropy, stats, top, top_logprob) if c["top_k"] else (logprob, entropy, stats)
        if c["op"] == "logp_grad":
            return B.bc_token_logprobs_backward(s["logits"], s["targets"], s["stats"], s["entropy"], s["d_logprob"], s["d_entropy"])
        if c["op"] == "norm":
            return B.bc_block_norm(s["x"], s["h"], s["gate"], s["post_weight"], s["pre_weight"], EPS, c["scale"], c["post"])
        if c["op"] == "norm_grad":
            dx, dh, dgate, dpost, dpre = B.bc_block_norm_backward(s["x"], s["h"], s["gate"], s["post_weight"], s["pre_weight"], EPS,
                                                                  c["scale"], c["post"], s["dh"], s["dy"])
            return [t for t in (dx, dh, dpre, dpost, dgate) if t is not None]
        return B.bc_mask_attn_backward(s["prompt_lens"], s["token_lens"], c["c"], s["prompt_k"], s["prompt_v"], s["tok_q"], s["tok_k"],
                                       s["tok_v"], s["beacon_q"], s["beacon_k"], s["beacon_v"], s["out_tok"], s["out_beacon"],
                                       s["lse_tok"], s["lse_beacon"], s["d_tok"], s["d_beacon"], s["scale"], check=False)
    if c["op"] == "logp":
        return _logp_plain(s)
    if c["op"] == "logp_grad":
        return _logp_grad_plain(s)
    if c["op"] == "norm":
        return _block_norm(s)
    if c["op"] == "norm_grad":
        return _block_norm_grad(s)
    return _mask_grad_plain(s)


def work(case):
    n = case["n"]
    if case["op"] in ("logp", "logp_grad"):
        v, size = case["vocab"], 4 if case["f32"] else 2
        if case["op"] == "logp":
            return dict(bytes=n * v * size + n * (8 + 16 + 8 * case["top_k"]), flops=5 * n * v)
        return dict(bytes=2 * n * v * size + n * (8 + 20), flops=6 * n * v)
    if case["op"] in ("norm", "norm_grad"):
        h, gate, post = case["hidden"], case["gate"], case["post"]
        once = (1 + post + (gate == "vector")) * 2 * h                    # the vectors
        rows = n * h * 2 * (gate == "rows")
        if case["op"] == "norm":
            return dict(bytes=8 * n * h + rows + once, flops=(6 + 4 * post) * n * h)
        return dict(bytes=12 * n * h + 2 * rows + once + 4 * h * (1 + post + (gate == "vector")), flops=(12 + 12 * post) * n * h)
    p, t, nb = _lengths(case)
    hq, hk, c = case["q_heads"], case["kv_heads"], case["c"]
    pairs = 0
    for P, T, N in zip(p, t, nb):
        own_rows = T * (T + 1) // 2 if c == 1 else N * (c * (c + 1) // 2) + (T % c) * (T % c + 1) // 2
        before = 0 if c == 1 else c * N * (N - 1) // 2 + (T % c) * N      # beacons that token rows see
        pairs += (T + N) * P + own_rows + before + N * (N + 1) // 2 + N * c
    rows, keys = sum(t) + sum(nb), sum(p) + sum(t) + sum(nb)
    return dict(bytes=2 * 128 * (4 * rows * hq + 4 * keys * hk) + 4 * rows * hq, flops=10 * 128 * hq * pairs)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "logp":
        x = s["logits"].double()
        lp = torch.log_softmax(x, -1)
        p = lp.exp()
        entropy = -torch.xlogy(p, p).sum(-1)
        t = s["targets"]
        given = torch.where(t >= 0, lp[torch.arange(case["n"], device=DEV), t.clamp(min=0)], 0.0)
        best = x.max(-1).values
        out = [given, entropy, torch.stack([best, torch.logsumexp(x, -1) - best], 1)]
        if case["top_k"]:
            del p
            z = torch.sort(x, dim=-1, descending=True, stable=True)
            out += [z.indices[:, :case["top_k"]].int(), lp.gather(1, z.indices[:, :case["top_k"]])]
        return tuple(out)
    if case["op"] == "logp_grad":
        x = s["logits"].double()
        lp = torch.log_softmax(x, -1)
        p = lp.exp()
        entropy = -torch.xlogy(p, p).sum(-1, keepdim=True)
        g = torch.where(s["targets"] >= 0, s["d_logprob"].double(), 0.0)[:, None]
        grad = -(g * p + s["d_entropy"].double()[:, None] * (torch.xlogy(p, p) + p * entropy))
        rows = torch.arange(case["n"], device=DEV)
        grad[rows, s["targets"].clamp(min=0)] += g[:, 0]
        return grad
    if case["op"] in ("norm", "norm_grad"):
        to = lambda k: None if s[k] is None else s[k].double().requires_grad_()
        x, h, gate, post, pre = [to(k) for k in ("x", "h", "gate", "post_weight", "pre_weight")]
        unit = lambda y, w: y / torch.sqrt((y ** 2).sum(-1, keepdim=True) / case["hidden"] + EPS) * w
        u = (unit(x, post) if case["post"] else x) * case["scale"]
        u = u if gate is None else u * gate
        if case["op"] == "norm":
            new = (h + u).detach()
            return new, unit(new.to(torch.bfloat16).double(), pre).detach()
        # the residual stream is given as it was stored; what reaches it goes on to the block's output unchanged
        dz, dpre = torch.autograd.grad((unit(h, pre) * s["dy"].double()).sum(), (h, pre))
        dh = s["dh"].double() + dz
        leaves = [x] + ([post] if case["post"] else []) + ([] if gate is None else [gate])
        more = torch.autograd.grad((u * dh).sum(), leaves)
        return [more[0], dh, dpre] + list(more[1:])
    p, t, nb = _lengths(case)
    hq, hk, c, n = case["q_heads"], case["kv_heads"], case["c"], case["n"]
    if sum((a + b) * (a + b + e) for a, b, e in zip(t, nb, p)) * hq > 1.2e10:
        return None
    names = ("prompt_k", "prompt_v", "tok_q", "tok_k", "tok_v", "beacon_q", "beacon_k", "beacon_v")
    out = {k: torch.zeros(s[k].shape, dtype=torch.float64, device=DEV) for k in names}
    for i in range(n):
        cut = lambda ln: slice(sum(ln[:i]), sum(ln[:i + 1]))
        cp, ct, cb = cut(p), cut(t), cut(nb)
        P, T, N = p[i], t[i], nb[i]
        # who sees what, written out by the definition: a row per token and beacon, a column per prompt entry, beacon and token
        see = torch.zeros((T + N, P + N + T), dtype=torch.bool, device=DEV)
        see[:, :P] = True
        tok = torch.arange(T, device=DEV)
        if c == 1:
            see[:, P:] = tok[None, :] <= tok[:, None]
        else:
            bea = torch.arange(N, device=DEV)
            see[:T, P:P + N] = (bea[None, :] + 1) * c <= tok[:, None]
            see[:T, P + N:] = (tok[None, :] <= tok[:, None]) & (tok[None, :] >= tok[:, None] - tok[:, None] % c)
            see[T:, P:P + N] = bea[None, :] <= bea[:, None]
            see[T:, P + N:] = (tok[None, :] >= bea[:, None] * c) & (tok[None, :] < (bea[:, None] + 1) * c)
        for h in range(hq):
            j = h * hk // hq
            q = torch.cat([s["tok_q"][ct, h], s["beacon_q"][cb, h]]).double()
            k = torch.cat([s["prompt_k"][cp, j], s["beacon_k"][cb, j], s["tok_k"][ct, j]]).double()
            v = torch.cat([s["prompt_v"][cp, j], s["beacon_v"][cb, j], s["tok_v"][ct, j]]).double()
            do = torch.cat([s["d_tok"][ct, h], s["d_beacon"][cb, h]]).double()
            a = torch.softmax((q @ k.T / math.sqrt(128)).masked_fill(~see, -math.inf), -1)
            da = do @ v.T
            dz = a * (da - (a @ v * do).sum(-1, keepdim=True)) / math.sqrt(128)
            dq, dk, dv = dz @ k, dz.T @ q, a.T @ do
            out["tok_q"][ct, h] += dq[:T]
            out["beacon_q"][cb, h] += dq[T:]
            for name, g in (("k", dk), ("v", dv)):
                out["prompt_" + name][cp, j] += g[:P]
                out["beacon_" + name][cb, j] += g[P:P + N]
                out["tok_" + name][ct, j] += g[P + N:]
    return tuple(out[k] for k in names)
