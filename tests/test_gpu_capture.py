"""Gate and adjudication captured into CUDA graphs and mixed with other calls on the same context."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _ctx():
    from paper_2608_02611_b200 import binding
    return binding, binding.Context(0)


def _tensors(n, k, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    ref = torch.randn(n, generator=g, device=DEV).to(torch.bfloat16)
    cands = []
    for i in range(k):
        c = ref.clone()
        c[i::97 + i] += 1.0                    # i-dependent numbers of mismatches
        cands.append(c)
    return ref, cands


def _capture(call):
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    return graph, out


def test_replays_after_the_workspaces_have_been_outgrown():
    """A captured gate call and a captured adjudication still give their records after calls with more
    candidates and more timings have outgrown both workspaces."""
    kb, ctx = _ctx()
    ctx.set_small_path(False)
    ref, cands = _tensors(1 << 16, 5, 1)
    t = torch.rand(40, 200, device=DEV) + 1.0
    want = kb.records(ctx.screen(ref, cands, 1e-2, 1e-2)).tobytes()
    median, iqr, wins = [v.clone() for v in ctx.adjudicate(t)]
    graph, (out, adj) = _capture(lambda: (ctx.screen(ref, cands, 1e-2, 1e-2), ctx.adjudicate(t)))
    for K in (1500, 5000):
        ctx.screen(ref, [cands[i % 5] for i in range(K)], 1e-2, 1e-2)
        ctx.adjudicate(torch.rand(K // 10, 1000, device=DEV) + 1.0)
        held = torch.full((32 << 20,), 7.0, device=DEV)
        out.fill_(0xEE)
        graph.replay()
        torch.cuda.synchronize()
        assert kb.records(out).tobytes() == want
        for got, same in zip(adj, (median, iqr, wins)):
            assert bool((got == same).all())
        assert bool((held == 7.0).all())
        del held
    assert ctx.poll() == 0 and ctx.check_guards()[1] == 0
    del graph, out, adj
    ctx.close()


@pytest.mark.parametrize("dtype,small", [(torch.bfloat16, False), (torch.float8_e4m3fn, False), (torch.float64, False),
                                         (torch.bfloat16, True)])
def test_calls_between_replays_give_their_own_records(dtype, small):
    """Replays and direct calls in turn, with numbers of candidates that differ: neither leaves anything behind
    in the accumulators for the other."""
    kb, ctx = _ctx()
    ctx.set_small_path(small)
    ref, cands = _tensors(1 << 16, 12, 2)
    ref, cands = ref.to(dtype), [c.to(dtype) for c in cands]
    screen, records = (ctx.screen_f64, kb.records_f64) if dtype == torch.float64 else (ctx.screen, kb.records)
    fresh = kb.Context(0)
    fresh.set_small_path(small)
    one = fresh.screen_f64 if dtype == torch.float64 else fresh.screen
    few, many = [records(one(ref, c, 1e-2, 1e-2)).tobytes() for c in (cands[:3], cands)]
    fresh.close()
    screen(ref, cands, 1e-2, 1e-2)
    graph, out = _capture(lambda: screen(ref, cands, 1e-2, 1e-2))
    for order in ("mrf", "rmfr", "frfm", "rrm", "mfrmrrfmffrrfrmfm"):
        for step in order:
            if step == "r":
                graph.replay()
                torch.cuda.synchronize()
            got = {"r": lambda: out, "f": lambda: screen(ref, cands[:3], 1e-2, 1e-2),
                   "m": lambda: screen(ref, cands, 1e-2, 1e-2)}[step]()
            assert records(got).tobytes() == (few if step == "f" else many), (order, step)
    assert ctx.poll() == 0
    del graph, out
    ctx.close()


def test_growth_of_the_gates_workspace_inside_a_capture_is_refused():
    kb, ctx = _ctx()
    ctx.set_small_path(False)
    ref, cands = _tensors(4096, 2, 3)
    many = [cands[i % 2] for i in range(3000)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(kb.KbError) as e:
        with torch.cuda.graph(graph):
            ctx.screen(ref, many, 1e-2, 1e-2)
    assert e.value.status == 4
    want = kb.records(ctx.screen(ref, many, 1e-2, 1e-2)).tobytes()
    graph, out = _capture(lambda: ctx.screen(ref, many, 1e-2, 1e-2))
    graph.replay()
    torch.cuda.synchronize()
    assert kb.records(out).tobytes() == want
    del graph, out
    ctx.close()


def test_first_adjudication_inside_a_capture_counts_without_a_workspace():
    kb, ctx = _ctx()
    t = torch.rand(40, 200, device=DEV) + 1.0
    graph, adj = _capture(lambda: ctx.adjudicate(t))
    graph.replay()
    torch.cuda.synchronize()
    held = [v.clone() for v in adj]
    for got, want in zip(held, ctx.adjudicate(t)):
        assert bool((got == want).all())
    assert ctx.poll() == 0
    del graph, adj
    ctx.close()
