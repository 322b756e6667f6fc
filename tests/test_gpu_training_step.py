"""The training operators together, as a student's layer uses them on compressed trajectories: norm and rotation of the heads, the mask
form, the norms around the block, log-probabilities and distillation -- and every gradient back through them, against the same chain
in fp64 autograd.  The products between them are PyTorch's."""
import math

import pytest
import torch

from paper_2510_13797_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
EPS = 1e-6
BF16, F64 = torch.bfloat16, torch.float64


def _rand(g, *shape, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(BF16)


def _rms(x, w):
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * w


def _rope(x, pos, theta):
    d = x.shape[-1]
    a = pos.to(F64)[:, None, None] * theta ** (-2.0 * torch.arange(d // 2, dtype=F64, device=DEV) / d)
    lo, hi = x[..., :d // 2], x[..., d // 2:]
    return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1)


def _visible(P, T, c):
    nb = T // c
    r, k = torch.arange(T + nb, device=DEV)[:, None], torch.arange(P + nb + T, device=DEV)[None]
    is_b = r >= T
    w = torch.where(is_b, r - T, r // c)
    tok = k - P - nb
    return (k < P) | ((k >= P) & (tok < 0) & (k - P < w + is_b)) | ((tok >= 0) & (tok // c == w) & (is_b | (tok <= r)))


def test_a_layer_forward_and_backward():
    P, T, c, Hq, Hkv, D, hidden, vocab = [37, 90], [200, 131], 8, 8, 2, 128, 512, 3001
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    nb = [t // c for t in T]
    st, sb = sum(T), sum(nb)
    rows, width, scale = st + sb, (Hq + 2 * Hkv) * D, 1 / math.sqrt(D)
    h, prompt_k, prompt_v = _rand(g, rows, hidden, scale=2.0), _rand(g, sum(P), Hkv, D), _rand(g, sum(P), Hkv, D)
    wqkv, wo, head = _rand(g, hidden, width, scale=hidden ** -0.5), _rand(g, Hq * D, hidden, scale=(Hq * D) ** -0.5), _rand(g, hidden, vocab, scale=0.1)
    w0, w1, w2, qw, kw = [1 + _rand(g, n, scale=0.1) for n in (hidden, hidden, hidden, D, D)]
    gate = 1 + _rand(g, hidden, scale=0.2)
    pos = torch.randint(0, 2000, (rows,), generator=g, device=DEV, dtype=torch.int32)
    targets = torch.randint(0, vocab, (st,), generator=g, device=DEV)
    targets[::7] = -100
    gl, ge = torch.randn(st, generator=g, device=DEV), 0.2 * torch.randn(st, generator=g, device=DEV)
    teacher = torch.randn((st, vocab), generator=g, device=DEV).to(BF16) * 3

    # ---- the library's chain
    _, y0 = B.bc_block_norm(torch.zeros_like(h), h, None, None, w0, EPS, 1.0, False)
    qkv = y0 @ wqkv
    q, k, v = B.bc_norm_rope_split(qkv, pos, 1e4, qw, kw, EPS, Hq, Hkv)
    cut = lambda t: (t[:st].contiguous(), t[st:].contiguous())
    (tq, bq), (tk, bk), (tv, bv) = cut(q), cut(k), cut(v)
    ins = (prompt_k, prompt_v, tq, tk, tv, bq, bk, bv)
    out = B.bc_mask_attn_forward_lse(P, T, c, *ins, scale)
    att = torch.cat(out[:2]).view(rows, Hq * D)
    x = att @ wo
    h1, y1 = B.bc_block_norm(x, h, gate, w1, w2, EPS, 0.5, True)
    logits = y1[:st] @ head
    logprob, entropy, stats, _, _ = B.bc_token_logprobs(logits, targets)
    _, _, _, idx, top = B.bc_token_logprobs(teacher, None, 50)
    cu = torch.tensor([0, T[0], st], dtype=torch.int32, device=DEV)
    kl, _, d_kl = B.bc_distill_loss(cu, logits, idx, top, with_grad=True)
    loss = (gl * logprob).sum() + (ge * entropy).sum() + 50 * kl
    d_logits = (B.bc_token_logprobs_backward(logits, targets, stats, entropy, gl, ge).float() + 50 * d_kl.float()).to(BF16)
    d_head = y1[:st].t().float() @ d_logits.float()
    dy1 = torch.cat([d_logits @ head.t(), torch.zeros((sb, hidden), dtype=BF16, device=DEV)])
    dx, dh, d_gate, d_w1, d_w2 = B.bc_block_norm_backward(x, h1, gate, w1, w2, EPS, 0.5, True, None, dy1)
    d_wo = att.t().float() @ dx.float()
    d_tok, d_bea = cut((dx @ wo.t()).view(rows, Hq, D))
    grads = B.bc_mask_attn_backward(P, T, c, *ins, *out, d_tok, d_bea, scale)
    dq, dk, dv = (torch.cat([grads[i], grads[i + 3]]) for i in (2, 3, 4))
    dqkv, d_qw, d_kw = B.bc_norm_rope_split_backward(qkv, pos, 1e4, qw, kw, EPS, dq, dk, dv)
    d_wqkv = y0.t().float() @ dqkv.float()
    _, dh0, _, _, d_w0 = B.bc_block_norm_backward(torch.zeros_like(h), h, None, None, w0, EPS, 1.0, False, dh, dqkv @ wqkv.t())
    got = dict(h=dh0, prompt_k=grads[0], prompt_v=grads[1], wqkv=d_wqkv, wo=d_wo, head=d_head, w0=d_w0, w1=d_w1, w2=d_w2, qw=d_qw, kw=d_kw, gate=d_gate)

    # ---- the same in 64 bits
    par = dict(h=h, prompt_k=prompt_k, prompt_v=prompt_v, wqkv=wqkv, wo=wo, head=head, w0=w0, w1=w1, w2=w2, qw=qw, kw=kw, gate=gate)
    z = {n: t.to(F64).requires_grad_() for n, t in par.items()}
    s = (_rms(z["h"], z["w0"]) @ z["wqkv"]).view(rows, Hq + 2 * Hkv, D)
    q, k, v = _rope(_rms(s[:, :Hq], z["qw"]), pos, 1e4), _rope(_rms(s[:, Hq:Hq + Hkv], z["kw"]), pos, 1e4), s[:, Hq + Hkv:]
    att = torch.zeros((rows, Hq, D), dtype=F64, device=DEV)
    for i in range(2):
        a, b, e = slice(sum(P[:i]), sum(P[:i + 1])), slice(sum(T[:i]), sum(T[:i + 1])), slice(st + sum(nb[:i]), st + sum(nb[:i + 1]))
        see = _visible(P[i], T[i], c)
        kk, vv = torch.cat([z["prompt_k"][a], k[e], k[b]]), torch.cat([z["prompt_v"][a], v[e], v[b]])
        kk, vv = [t.repeat_interleave(Hq // Hkv, 1) for t in (kk, vv)]
        w = torch.einsum("rhd,khd->hrk", torch.cat([q[b], q[e]]), kk) * scale
        o = torch.einsum("hrk,khd->rhd", w.masked_fill(~see, -math.inf).softmax(-1), vv)
        att = att.index_add(0, torch.cat([torch.arange(rows, device=DEV)[b], torch.arange(rows, device=DEV)[e]]), o)
    y = _rms(z["h"] + 0.5 * z["gate"] * _rms(att.reshape(rows, Hq * D) @ z["wo"], z["w1"]), z["w2"])
    lp = torch.log_softmax(y[:st] @ z["head"], -1)
    given = torch.where(targets >= 0, lp[torch.arange(st, device=DEV), targets.clamp(min=0)], 0.0)
    tp = top.to(F64)
    row = (tp.exp() * (tp - lp.gather(1, idx.long()))).sum(-1)
    want_loss = (gl.to(F64) * given).sum() - (ge.to(F64) * (lp.exp() * lp).sum(-1)).sum() + 50 * (row[:T[0]].mean() + row[T[0]:].mean()) / 2
    want = dict(zip(z, torch.autograd.grad(want_loss, list(z.values()))))
    # Some twenty tensors are rounded to bf16 between a parameter and its gradient, each off by 2^-8 of itself at most and none magnified:
    # relative to the gradient as a whole 20 * 2^-8 at most.  (The loss: its logits, in the same way.)
    for n in par:
        off = (got[n].to(F64) - want[n]).norm() / want[n].norm()
        assert off <= 20 * 2.0 ** -8, (n, float(off))
    size = (gl.abs() * logprob.abs()).sum() + (ge.abs() * entropy).sum() + 50 * kl.abs()
    assert abs(float(loss) - float(want_loss.detach())) <= 20 * 2.0 ** -8 * float(size)


def _calls():
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    x = _rand(g, 64, 5000)
    t = torch.randint(0, 5000, (64,), generator=g, device=DEV)
    one = torch.ones(64, device=DEV)
    _, entropy, stats, _, _ = B.bc_token_logprobs(x, t)
    a, b, w = _rand(g, 300, 512), _rand(g, 300, 512), 1 + _rand(g, 512, scale=0.1)
    q, k, bq, bk = _rand(g, 60, 4, 128), _rand(g, 60, 2, 128), _rand(g, 15, 4, 128), _rand(g, 15, 2, 128)
    ins = ([0], [60], 4, None, None, q, k, k, bq, bk, bk)
    out = B.bc_mask_attn_forward_lse(*ins, 0.1)
    return {
        "logprobs": lambda **kw: B.bc_token_logprobs(x, t, 20, **kw),
        "logprobs_backward": lambda **kw: (B.bc_token_logprobs_backward(x, t, stats, entropy, one, one, **kw),),
        "block_norm": lambda **kw: B.bc_block_norm(a, b, w, w, w, EPS, **kw),
        "block_norm_backward": lambda **kw: B.bc_block_norm_backward(a, b, w, w, w, EPS, 1.0, True, a, b, **kw),
        "mask_lse": lambda **kw: B.bc_mask_attn_forward_lse(*ins, 0.1, check=False, **kw),
        "mask_backward": lambda **kw: B.bc_mask_attn_backward(*ins, *out, q, bq, 0.1, check=False, **kw)[2:],
    }


NAMES = ["logprobs", "logprobs_backward", "block_norm", "block_norm_backward", "mask_lse", "mask_backward"]


@pytest.mark.parametrize("name", NAMES)
def test_on_a_given_stream_with_results_of_its_own_memory(name):
    call = _calls()[name]
    want = call()
    sizes = [t.untyped_storage().nbytes() for t in want]
    s = torch.cuda.Stream()
    torch.cuda._sleep(1)
    torch.empty(8, dtype=torch.uint8, device=DEV).fill_(0)
    torch.cuda.synchronize()
    blocks = [torch.empty(size, dtype=torch.uint8, device=DEV) for size in sizes for _ in range(100)]
    torch.cuda._sleep(100_000_000)                       # some 50 ms; the writes behind it come after the call on the other stream
    for b in blocks:
        b.fill_(77)
    held = blocks[::2]
    del blocks, b                                        # free for the current stream, whose order protects them there
    got = call(stream=s)
    s.synchronize()
    first = [t.clone() for t in got]
    torch.cuda.synchronize()
    del held
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, got, first))


@pytest.mark.parametrize("name", NAMES)
def test_two_calls_at_once(name):
    call = _calls()[name]
    want = call()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [call(stream=streams[i % 2]) for i in range(8)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for r in got for a, b in zip(want, r))


def test_the_mask_form_with_its_gradient_refuses_capture():
    """Its work lists are copied from host memory that a replay would not find."""
    calls = _calls()
    graph = torch.cuda.CUDAGraph()
    y = torch.zeros(4, device=DEV)
    with torch.cuda.graph(graph):
        y += 1
        for name in ("mask_lse", "mask_backward"):
            with pytest.raises(B.BreadcrumbsError) as e:
                calls[name]()
            assert e.value.status == B.BC_ERR_UNSUPPORTED
    graph.replay()
    torch.cuda.synchronize()
    assert float(y[0]) == 1
