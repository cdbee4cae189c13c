"""The model operators captured into CUDA graphs: results of replays, and the workspace of the norm's backward
pass, whose address a captured launch keeps."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _context():
    from paper_2608_02611_b200 import binding
    return binding.Context(0), binding.KbError


def _inputs(rows, cols, seed, dtype=torch.bfloat16):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x, dy = (torch.randn(rows, cols, generator=g, device=DEV).to(dtype) for _ in range(2))
    w = torch.rand(cols, generator=g, device=DEV).to(dtype)
    m = x.float().mean(1)
    r = (x.float().var(1, unbiased=False) + 1e-5).rsqrt()
    return dy, x, w, m, r


def _captured(call):
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    return graph, out


def _same(got, want):
    return all(bool((a == b).all()) for a, b in zip(got, want))


def test_replay_after_the_workspace_has_been_outgrown():
    """A small backward pass is captured, larger ones outgrow its workspace twice, and the replays between and
    after them still give the small pass's gradients, on new inputs too."""
    ctx, _ = _context()
    small = _inputs(300, 512, 1)
    want = ctx.layernorm_backward(*small)
    graph, out = _captured(lambda: ctx.layernorm_backward(*small))
    for k, (rows, cols) in enumerate(((2000, 4096), (3000, 8192))):
        big = _inputs(rows, cols, 2 + k)
        first = ctx.layernorm_backward(*big)
        fill = torch.full((64 << 20,), float("nan"), device=DEV)      # whatever was freed may be handed out again
        for o in out:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert _same(out, want)
        assert _same(ctx.layernorm_backward(*big), first)
        assert bool(fill.isnan().all())
        del fill
        other = _inputs(300, 512, 7 + k)
        want = ctx.layernorm_backward(*other)
        for held, new in zip(small, other):
            held.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert _same(out, want)
    assert ctx.poll() == 0 and ctx.check_guards()[1] == 0
    del graph, out
    ctx.close()


@pytest.mark.parametrize("rows,cols", [(40, 384), (500, 1024), (9, 20000)])
def test_growth_inside_a_capture_is_refused_and_reserved_room_suffices(rows, cols):
    ctx, KbError = _context()
    args = _inputs(rows, cols, rows)
    launches = ctx.launch_count
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(KbError) as e:
        with torch.cuda.graph(graph):
            ctx.layernorm_backward(*args)
    assert e.value.status == 4 and "reserve" in str(e.value)
    assert ctx.launch_count == launches                            # nothing of the call was captured
    torch.cuda.synchronize()
    ctx.reserve_layernorm_backward(rows, cols)
    graph, out = _captured(lambda: ctx.layernorm_backward(*args))
    graph.replay()
    torch.cuda.synchronize()
    assert _same(out, ctx.layernorm_backward(*args))
    with pytest.raises(KbError):
        ctx.reserve_layernorm_backward(rows, 0)
    del graph, out
    ctx.close()


@pytest.mark.parametrize("cols", [1, 256, 512, 513, 768, 1000, 1024, 2056, 4096, 6144, 8192, 8200, 30000])
def test_reserved_room_covers_every_kernel(cols):
    """After a reservation for the most rows no backward pass over as many or fewer grows the workspace, aligned
    or not: no further allocation is let through."""
    ctx, _ = _context()
    most = max(1, min(5000, (1 << 24) // cols))
    ctx.reserve_layernorm_backward(most, cols)
    ctx.fail_next_allocs(1000)
    for dtype in (torch.bfloat16, torch.float32):
        for rows in sorted({1, 7, 100, 295, 296, 700, 1184, 2400, most}):
            if rows <= most:
                dy, x, w, m, r = _inputs(rows, cols, rows, dtype)
                ctx.layernorm_backward(dy, x, w, m, r)
                apart = torch.empty(rows, cols + 1, dtype=dtype, device=DEV)[:, :cols]
                apart.copy_(x)
                ctx.layernorm_backward(dy, apart, w, m, r)
    ctx.fail_next_allocs(0)
    assert ctx.poll() == 0
    ctx.close()


def test_first_calls_inside_a_capture():
    """A new context's first norm, quantisation and products, captured and replayed on new inputs."""
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x = torch.randn(200, 640, generator=g, device=DEV).to(torch.bfloat16)
    w = torch.rand(640, generator=g, device=DEV).to(torch.bfloat16)
    W = torch.randn(3000, 640, generator=g, device=DEV).to(torch.bfloat16)
    E4M3 = torch.float8_e4m3fn

    def step(ctx):
        h = ctx.layernorm(x, w, None, quantize=E4M3)
        q, s = ctx.quantize_blocks(W, tiles=True)
        qt, st = ctx.quantize_blocks(W, transpose=True)
        big, bs = ctx.quantize_blocks(W)
        return (h.y, h.mean, h.rstd, h.scale, s, st, ctx.matmul_blocks(h.q, h.scale, q, s), ctx.matmul_blocks(h.q[:1], h.scale[:, :1].contiguous(), q, s),
                ctx.matmul_blocks(big, bs, q, s), qt.float())

    ctx, _ = _context()
    graph, out = _captured(lambda: step(ctx))
    assert ctx.last_product == (256, 1)
    other, _ = _context()
    for k in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert _same(out, step(other))
        x.copy_(torch.randn(200, 640, generator=g, device=DEV))
        W.mul_(0.5)
    assert ctx.poll() == 0 and other.poll() == 0
    del graph, out
    ctx.close()
    other.close()
