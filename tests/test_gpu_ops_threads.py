"""The model operators called from several host threads, each with a context and a stream of its own."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_backward_passes_of_two_widths_in_two_threads():
    """Both take the walk through shared memory, with rings of different sizes (196 KB and 48 KB), through the
    same kernel: neither thread's call may lower the limit the other's launch needs."""
    from paper_2608_02611_b200 import binding
    L = binding.load()
    refused, calls = [], 4000
    barrier = threading.Barrier(2)

    def work(rows, cols):
        ctx = binding.Context(0)
        stream = torch.cuda.Stream()
        x = torch.randn(rows, cols, device=DEV).to(torch.bfloat16)
        mean, rstd, dx, dw = x.float().mean(1), torch.ones(rows, device=DEV), torch.empty_like(x), torch.empty(cols, device=DEV)
        torch.cuda.synchronize()
        want = ctx.layernorm_backward(x, x, None, mean, rstd)
        torch.cuda.synchronize()
        args = (ctx._h, x.data_ptr(), cols, x.data_ptr(), cols, rows, cols, binding.KB_BF16, None, binding.KB_F32,
                mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(), cols, dw.data_ptr(), None, stream.cuda_stream)
        barrier.wait()
        for i in range(calls):
            rc = L.kb_layernorm_backward(*args)
            if rc != 0:
                refused.append((cols, rc, L.kb_last_error(ctx._h)))
                break
            if i % 64 == 63:
                stream.synchronize()
        stream.synchronize()
        if not (bool((dx == want[0]).all()) and bool((dw == want[1]).all())):
            refused.append((cols, "other gradients"))
        if ctx.poll() != 0:
            refused.append((cols, "status"))
        ctx.close()

    threads = [threading.Thread(target=work, args=a) for a in ((300, 8192), (1200, 2048))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not refused, refused
