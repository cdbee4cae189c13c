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


WAIT_C = """
#include <time.h>
/* Stands in for any entry point: waits up to 5 s for another thread to set the flag. */
volatile int flag = 0;
int wait_for_flag(void) {
  for (int i = 0; i < 5000 && !flag; ++i) {
    struct timespec t = {0, 1000000};
    nanosleep(&t, 0);
  }
  return flag ? 0 : 5;
}
const char* no_error(const void* ctx) { return "the other thread did not run"; }
"""


def test_other_threads_run_while_an_operator_call_waits(tmp_path):
    """A call whose entry point waits (here a stand-in on the host; no kernel runs) leaves Python's lock to the
    other threads, one of which ends the wait."""
    import ctypes
    import subprocess
    from paper_2608_02611_b200 import binding
    src, lib = tmp_path / "wait.c", tmp_path / "wait.so"
    src.write_text(WAIT_C)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(lib), str(src)], check=True)
    W = ctypes.CDLL(str(lib))
    flag = ctypes.c_int.in_dll(W, "flag")
    wait, text = (ctypes.cast(f, ctypes.c_void_p).value for f in (W.wait_for_flag, W.no_error))
    ctx = binding.Context(0)
    x = torch.randn(64, 256, device=DEV)
    m, r = torch.zeros(64, device=DEV), torch.ones(64, device=DEV)
    q, s = ctx.quantize_blocks(x)
    calls = (lambda: ctx.quantize_blocks(x), lambda: ctx.layernorm(x), lambda: ctx.layernorm_backward(x, x, None, m, r),
             lambda: ctx.matmul_blocks(q, s, q, s))
    module = binding._native()
    module.bind(binding.KbError, wait, wait, wait, wait, text)
    try:
        for call in calls:
            flag.value = 0
            started = threading.Event()

            def release():
                started.wait()
                flag.value = 1

            t = threading.Thread(target=release)
            t.start()
            started.set()
            try:
                call()                    # KbError if the flag was not set meanwhile
            finally:
                t.join()
    finally:
        binding._native_module = None     # the library's own entry points again
        binding._native()
    assert bool((ctx.quantize_blocks(x)[1] == s).all())
    ctx.close()
