"""Values that are not finite in prompts: they reach the queries that see them, in their own places, and nothing else.

A call with such values is compared with the same call with zeros in their place: bit for bit wherever no such value is
seen; where some are, their sum with anything finite is what the definition gives, whatever their probabilities."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
HALVES = [torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def ctx():
    from paper_2608_02611_b200 import binding
    c = binding.Context(0)
    yield c
    assert c.poll() == 0
    assert c.check_guards()[1] == 0
    c.close()


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def _offsets(lens):
    return torch.tensor([0] + list(lens)).cumsum(0).to(torch.int32).to(DEV)


def _seen_sums(v, qlens, klens, causal, group):
    """Per query, head and element the sum of the values it sees that are not finite; 0 where there are none."""
    odd = torch.where(v.double().isfinite(), 0.0, v.double())
    parts, at = [], 0
    for nq, nk in zip(qlens, klens):
        upto = torch.cat([torch.zeros_like(odd[:1]), odd[at:at + nk].cumsum(0)])   # of the first 0, 1, .. keys
        seen = (torch.arange(nq) + 1 + nk - nq).clamp(0, nk) if causal else torch.full((nq,), nk)
        parts.append(upto[seen])
        at += nk
    return torch.cat(parts).repeat_interleave(group, 1)


def _check(ctx, q, k, v, qlens, klens, causal):
    args = [_offsets(qlens), _offsets(klens)]
    zeroed = torch.where(v.isfinite(), v, torch.zeros_like(v))
    got, want = (ctx.attention(q.to(DEV), k.to(DEV), x.to(DEV), *args, causal=causal, want_lse=True) for x in (v, zeroed))
    assert ctx.poll() == 0
    sums = _seen_sums(v, qlens, klens, causal, q.shape[1] // k.shape[1])
    out, clean = got.out.cpu(), want.out.cpu()
    assert torch.equal(got.lse, want.lse) and bool(clean.isfinite().all())
    none = sums == 0.0
    assert torch.equal(out[none].view(torch.int16), clean[none].view(torch.int16))
    assert torch.equal(out[sums.isnan()].isnan(), torch.ones(int(sums.isnan().sum()), dtype=torch.bool))
    for sign in (1, -1):
        assert bool((out[sums == sign * math.inf] == sign * math.inf).all())


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("hq,hkv,dim", [(2, 1, 128), (3, 1, 64), (1, 1, 72), (320, 160, 64), (165, 165, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_each_value_reaches_who_sees_it_and_nobody_else(ctx, dtype, hq, hkv, dim, causal):
    """One and two heads of a group and two pieces at a time (few and many heads, odd and even groups), lengths that end
    inside steps, pieces whose first step that is looked at begins inside another's."""
    qlens = [1, 64, 65, 127, 129, 256, 300, 0, 100, 50, 5]
    klens = [1, 64, 65, 127, 200, 300, 333, 3, 900, 20, 0]
    gen = _gen(hq + dim)
    n = sum(klens)
    q = torch.randn(sum(qlens), hq, dim, generator=gen).to(dtype)
    k, v = (torch.randn(n, hkv, dim, generator=gen).to(dtype) for _ in range(2))
    for i in range(60):
        t, d = (int(torch.randint(m, (1,), generator=gen)) for m in (n, dim))
        v[t, i % hkv, d] = (math.nan, math.inf, -math.inf)[i % 3]
    v[n - 905:n - 900, 0] = math.inf     # whole rows, one behind another
    _check(ctx, q, k, v, qlens, klens, causal)


@pytest.mark.parametrize("dtype", HALVES)
def test_no_value_that_is_finite(ctx, dtype):
    q, k = (torch.randn(700, h, 64, generator=_gen(h)).to(dtype) for h in (4, 2))
    for x in (math.nan, math.inf):
        _check(ctx, q, k, torch.full((700, 2, 64), x, dtype=dtype), [300, 400], [200, 500], True)


@pytest.mark.parametrize("n,hq,dim", [(16384, 8, 128), (70001, 2, 64), (131072, 2, 128), (131072, 3, 64)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_late_in_long_texts(ctx, n, hq, dim, bad):
    """One value near the end: nothing of the tokens before it changes, no wait runs out, and the call takes about as long
    as without (a factor of 3 leaves room for the clock; work that grew with the text would take hundreds)."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(n)
    q, k, v = (torch.randn(n, h, dim, generator=gen, device=DEV, dtype=torch.float32).to(torch.bfloat16) for h in (hq, 1, 1))
    at = n - 60
    v[at] = 0.0
    w = v.clone()
    w[at, 0, 5] = bad
    out = []
    times = []
    for x in (v, w):
        ctx.attention(q, k, x)
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        out.append(ctx.attention(q, k, x).out)
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b))
    assert ctx.poll() == 0
    assert bool((out[1][at:, :, 5].isnan() if math.isnan(bad) else out[1][at:, :, 5] == bad).all())
    out[1][at:, :, 5] = out[0][at:, :, 5]
    assert torch.equal(out[0].view(torch.int16), out[1].view(torch.int16))
    assert times[1] <= 3 * times[0] + 0.1, times
