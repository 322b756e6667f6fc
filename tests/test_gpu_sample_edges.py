"""bc_sample where host threads could make it go wrong."""
import threading

import pytest
import torch

from paper_2510_13797_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"


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
