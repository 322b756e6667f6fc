"""Results that the binding allocates itself for a call on a given stream: their memory may not be that of work still queued on the
current stream."""
import pytest
import torch

from paper_2510_13797_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _calls():
    n, Hq, Hkv, D = 64, 4, 2, 64
    qkv = torch.randn((n, (Hq + 2 * Hkv) * D), device=DEV).to(torch.bfloat16)
    pos, w = torch.arange(n, dtype=torch.int32, device=DEV), torch.ones(D, dtype=torch.bfloat16, device=DEV)
    grads = [torch.randn((n, h, D), device=DEV).to(torch.bfloat16) for h in (Hq, Hkv, Hkv)]
    x, u = torch.randn((n, 999), device=DEV), torch.rand(n, device=DEV)
    cache = B.Cache(1, Hkv, Hq, D, 1, 16, max_seqs=1, num_pages=8, max_pages_per_seq=8)
    slot, k = torch.zeros(1, dtype=torch.int32, device=DEV), torch.randn((40, Hkv, D), device=DEV).to(torch.bfloat16)
    cache.bc_seq_open(slot, slot + 40)
    cache.bc_prefill(0, slot, torch.tensor([0, 40], dtype=torch.int32, device=DEV), 40, k, k)
    mq, mk = torch.randn((60, 4, 128), device=DEV).to(torch.bfloat16), torch.randn((60, 2, 128), device=DEV).to(torch.bfloat16)
    cu, idx = torch.tensor([0, 64], dtype=torch.int32, device=DEV), torch.arange(5, dtype=torch.int32, device=DEV).repeat(64, 1)
    logp = torch.full((64, 5), -2.0, device=DEV)
    z = torch.randn((64, 1000), device=DEV).to(torch.bfloat16)
    return {
        "sample": lambda **kw: (B.bc_sample(x, u, **kw),),
        "split": lambda **kw: B.bc_norm_rope_split(qkv, pos, 1e4, w, w, 1e-6, Hq, Hkv, **kw),
        "backward": lambda **kw: B.bc_norm_rope_split_backward(qkv, pos, 1e4, w, w, 1e-6, *grads, **kw),
        "export": lambda **kw: cache.bc_export_seq(0, 0, 40, **kw),
        "mask": lambda **kw: B.bc_mask_attn_forward([0], [60], 4, None, None, mq, mk, mk, mq[:15], mk[:15], mk[:15], 0.1, check=False, **kw),
        "distill": lambda **kw: B.bc_distill_loss(cu, z, idx, logp, with_grad=True, **kw),
    }


@pytest.mark.parametrize("name", ["sample", "split", "backward", "export", "mask", "distill"])
def test_results_do_not_share_memory_with_work_on_the_current_stream(name):
    call = _calls()[name]
    want = call()
    sizes = [t.untyped_storage().nbytes() for t in want]
    s = torch.cuda.Stream()
    torch.cuda._sleep(1)                                 # kernels are loaded by their first launch, which may wait for the device
    torch.empty(8, dtype=torch.uint8, device=DEV).fill_(0)
    torch.cuda.synchronize()
    blocks = [torch.empty(size, dtype=torch.uint8, device=DEV) for size in sizes for _ in range(100)]
    torch.cuda._sleep(100_000_000)                       # some 50 ms; the writes behind it come after the call on the other stream
    for b in blocks:
        b.fill_(77)
    held = blocks[::2]                                   # so that the others stay apart
    del blocks, b                                        # free for the current stream, whose order protects them there
    got = call(stream=s)
    s.synchronize()
    first = [t.clone() for t in got]
    torch.cuda.synchronize()
    del held
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, got, first))


def test_any_object_with_a_stream_handle_is_a_stream():
    class Handle:
        def __init__(self, s):
            self.cuda_stream = s.cuda_stream

    s = torch.cuda.Stream()
    for call in _calls().values():
        want = call()
        torch.cuda.synchronize()
        got = call(stream=Handle(s))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    B.Cache(1, 2, 4, 64, 1, 16, max_seqs=1, num_pages=1, max_pages_per_seq=1, stream=Handle(s))
    torch.cuda.synchronize()


def test_a_cache_created_on_a_stream_does_not_share_memory_with_work_on_the_current_stream():
    Hkv, D = 2, 64
    make = lambda s: B.Cache(1, Hkv, 2 * Hkv, D, 1, 16, max_seqs=2, num_pages=20, max_pages_per_seq=8, stream=s)
    first = make(None)
    sizes = [first.pool_bytes, first.meta_bytes, first.workspace_bytes]
    slot, cu = torch.ones(1, dtype=torch.int32, device=DEV), torch.tensor([0, 40], dtype=torch.int32, device=DEV)
    plen, k = slot * 40, torch.randn((40, Hkv, D), device=DEV).to(torch.bfloat16)
    s = torch.cuda.Stream()
    torch.cuda._sleep(1)
    torch.empty(8, dtype=torch.uint8, device=DEV).fill_(0)
    torch.cuda.synchronize()
    blocks = [torch.empty(size, dtype=torch.uint8, device=DEV) for size in sizes for _ in range(2)]
    torch.cuda._sleep(100_000_000)
    for b in blocks:
        b.fill_(77)
    del blocks, b
    cache = make(s)
    s.synchronize()
    torch.cuda.synchronize()                             # what was queued has run; the cache is as it was made
    assert cache.bc_get_state(0) == first.bc_get_state(0)
    cache.bc_seq_open(slot, plen, stream=s)
    cache.bc_prefill(0, slot, cu, 40, k, k, stream=s)
    got = cache.bc_export_seq(0, 1, 40, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(x, k) for x in got) and cache.bc_poll_error()[0] == 0
