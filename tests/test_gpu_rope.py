"""Norms of queries and keys with the position rotation, against 64 bits (bounds: attention_exact.py)."""
import math

import pytest
import torch

from tests import attention_exact as exact

pytestmark = pytest.mark.gpu
DEV = "cuda"
FLOATS = [torch.float32, torch.float16, torch.bfloat16]


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


def _qkv(tokens, hq, hkv, dim, dtype, seed, offset=0):
    """Slices of one projection on the GPU, `offset` elements after an aligned address."""
    n = tokens * (hq + 2 * hkv) * dim
    held = torch.randn(n + offset, generator=_gen(seed)).to(dtype).to(DEV)
    x = held[offset:].view(tokens, hq + 2 * hkv, dim)
    return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]


def _freq(pairs, theta=1e4):
    return (theta ** (-torch.arange(pairs, dtype=torch.float64) / max(1, pairs))).to(DEV)


# dim, rotary dim: all lane counts, parts that are turned, pairs that are no multiple of 8 apart, odd dims
DIMS = [(8, 8), (16, 4), (20, 20), (64, 64), (64, 0), (80, 32), (96, 24), (100, 50), (128, 128), (128, 64), (129, 2), (192, 192), (256, 256), (7, 6), (1, 0)]


@pytest.mark.parametrize("dim,rot", DIMS)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", FLOATS)
def test_against_64_bits(ctx, dim, rot, interleaved, dtype):
    for tokens, hq, hkv, offset in ((1, 4, 1, 0), (37, 6, 3, 0), (5, 33, 11, 1)):
        q, k, _ = _qkv(tokens, hq, hkv, dim, dtype, dim * 100 + rot + tokens, offset)
        gen = _gen(dim + rot)
        wq, wk = (torch.rand(dim, generator=gen).add(0.5).to(dtype).to(DEV) for _ in range(2))
        pos = torch.randint(0, 5000, (tokens,), generator=gen).to(DEV)
        f = _freq(rot // 2) if rot else None
        before = q.clone()
        qo, ko = ctx.qk_norm_rope(q, k, pos if rot else None, f, wq, wk, 1e-5, interleaved=interleaved)
        assert torch.equal(q, before)
        for x, w, got, name in ((q, wq, qo, "q"), (k, wk, ko, "k")):
            want, bound = exact.rope(x, w, 1e-5, pos, f, interleaved)
            assert got.shape == x.shape and got.dtype == dtype
            exact.within(got, want, bound, f"{name} {tokens} x {x.shape[1]} x {dim}")


@pytest.mark.parametrize("dtype", FLOATS)
def test_without_norm_weights_or_rotation(ctx, dtype):
    q, k, _ = _qkv(9, 4, 2, 64, dtype, 3)
    pos = torch.arange(9).to(DEV)
    f = _freq(32)
    for norm in (True, False):
        qo, ko = ctx.qk_norm_rope(q, k, pos, f, eps=1e-6, norm=norm)
        want, bound = exact.rope(k, None, 1e-6 if norm else None, pos, f, False)
        exact.within(ko, want, bound, "k")
    qo, _ = ctx.qk_norm_rope(q, k, norm=False)
    assert torch.equal(qo, q)                      # nothing to do: the very same numbers
    wq = (torch.rand(64, generator=_gen(1)) + 0.5).to(DEV)
    qo, ko = ctx.qk_norm_rope(q, k, pos, f, wq, None)          # weights in binary32, one of them left out
    for x, w, got in ((q, wq, qo), (k, None, ko)):
        want, bound = exact.rope(x, w, 1e-6, pos, f, False)
        exact.within(got, want, bound)


def test_far_and_negative_positions_and_any_frequency(ctx):
    """The angle is reduced exactly: positions up to 2^40 and frequencies beyond a turn per position.  The 64-bit
    reference reduces pos * freq in whole numbers, where a double's product would have lost the fraction."""
    import fractions
    pos = torch.tensor([0, 1, -1, 10 ** 6, 2 ** 31 + 7, -2 ** 33 - 1, 2 ** 40 + 12345])
    f = torch.tensor([1.0, 0.3, 1e-4, 7.5, -2.25, 2.0 ** -30, 100.125, 3.14159], dtype=torch.float64)
    x = torch.randn(7, 1, 16, generator=_gen(5)).to(DEV)
    qo, _ = ctx.qk_norm_rope(x, x, pos.to(DEV), f.to(DEV), norm=False)
    two_pi = fractions.Fraction("6.283185307179586476925286766559005768394338798750211641949889")
    d = x.double().cpu()[:, 0]
    for t in range(7):
        for i in range(8):
            turns = fractions.Fraction(int(pos[t])) * fractions.Fraction(float(f[i])) / two_pi
            angle = float((turns - math.floor(turns)) * two_pi)
            a, b = float(d[t, i]), float(d[t, i + 8])
            # the part of a turn per position is good to 2^-53 of the frequency (at least of 1)
            tol = (abs(a) + abs(b)) * (8 * exact.U + 2.0 ** -49 * abs(int(pos[t])) * max(1.0, abs(float(f[i]))))
            assert abs(float(qo[t, 0, i]) - (a * math.cos(angle) - b * math.sin(angle))) <= tol, (t, i)
            assert abs(float(qo[t, 0, i + 8]) - (b * math.cos(angle) + a * math.sin(angle))) <= tol, (t, i)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("heads_first", [False, True])
def test_stores_in_a_paged_cache(ctx, dtype, heads_first):
    """Keys and values go to their slots, nothing else of the cache changes, negative slots store nothing."""
    tokens, hq, hkv, dim, pages, page = 700, 4, 2, 64, 50, 24
    q, k, v = _qkv(tokens, hq, hkv, dim, dtype, 11)
    shape = (pages, hkv, page, dim) if heads_first else (pages, page, hkv, dim)
    kc, vc = (torch.full(shape, 7.0 + i, dtype=dtype, device=DEV) for i in range(2))
    kv, vv = ((c.transpose(1, 2) if heads_first else c) for c in (kc, vc))
    slots = torch.randperm(pages * page, generator=_gen(2))[:tokens]
    slots[3] = slots[500] = -1
    pos = torch.arange(tokens)
    f = _freq(32)
    qo, ko = ctx.qk_norm_rope(q, k, pos.to(DEV), f, v=v, k_cache=kv, v_cache=vv, slots=slots.to(DEV))
    assert ctx.poll() == 0
    want_k, want_v = (torch.full((pages * page, hkv, dim), 7.0 + i, dtype=dtype) for i in range(2))
    kept = slots >= 0
    want_k[slots[kept]], want_v[slots[kept]] = ko.cpu()[kept], v.cpu()[kept]
    assert torch.equal(kv.cpu().reshape(-1, hkv, dim), want_k) and torch.equal(vv.cpu().reshape(-1, hkv, dim), want_v)
    # the cache alone, and without the queries
    kc2, vc2 = torch.zeros_like(kv), torch.zeros_like(vv)
    a, b = ctx.qk_norm_rope(q, k, pos.to(DEV), f, want_q=False, want_k=False, v=v, k_cache=kc2, v_cache=vc2, slots=slots.to(DEV))
    assert a is None and b is None
    assert torch.equal(kc2.cpu().reshape(-1, hkv, dim)[slots[kept]], ko.cpu()[kept])
    a, b = ctx.qk_norm_rope(q, k, pos.to(DEV), f, want_k=False)
    assert b is None and torch.equal(a, qo)


def test_slots_that_come_twice_hold_elements_of_their_tokens(ctx):
    """One after the other in the cache: slot 5 is everyone's, the others' neighbours stay as they were."""
    tokens = 3000
    q, k, v = _qkv(tokens, 2, 2, 64, torch.bfloat16, 3)
    kc, vc = (torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    _, ko = ctx.qk_norm_rope(q, k, v=v, k_cache=kc, v_cache=vc, slots=torch.full((tokens,), 5).to(DEV))
    for cache, rows in ((kc, ko), (vc, v)):
        assert bool((cache.view(32, 2, 64)[5] == rows).any(0).all())
        cache[0, 5] = 0
        assert not bool(cache.any())
    assert ctx.poll() == 0


def test_slots_that_are_not_there_store_nothing_and_show(ctx):
    q, k, v = _qkv(4, 2, 1, 64, torch.bfloat16, 1)
    kc, vc = torch.zeros(3, 16, 1, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(3, 16, 1, 64, dtype=torch.bfloat16, device=DEV)
    slots = torch.tensor([48, 5, 2 ** 40, -9]).to(DEV)
    ctx.qk_norm_rope(q, k, v=v, k_cache=kc, v_cache=vc, slots=slots)
    assert ctx.poll() == 1 and ctx.poll() == 0
    assert int(vc.ne(0).any(-1).sum()) == 1 and torch.equal(vc.view(48, 64)[5], v[1, 0])


@pytest.mark.parametrize("dim,rot", [(128, 128), (100, 50)])
def test_in_place_and_in_graphs(ctx, dim, rot):
    q, k, _ = _qkv(300, 5, 5, dim, torch.bfloat16, 9)
    pos, f = torch.arange(300).to(DEV), _freq(rot // 2)
    want = ctx.qk_norm_rope(q, k, pos, f)
    for captured in (False, True):
        a, b = q.clone(), k.clone()
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                got = ctx.qk_norm_rope(a, b, pos, f, out=(a, b))
            assert torch.equal(a, q)
            graph.replay()
        else:
            got = ctx.qk_norm_rope(a, b, pos, f, out=(a, b))
        assert got[0].data_ptr() == a.data_ptr()
        assert torch.equal(a, want[0]) and torch.equal(b, want[1])


def test_nan_and_infinity_stay_in_their_heads(ctx):
    q, k, _ = _qkv(6, 3, 3, 64, torch.float32, 4)
    q, k = q.clone(), k.clone()
    want = ctx.qk_norm_rope(q, k, norm=True)[0]
    q[2, 1, 5], q[4, 0, 63] = float("nan"), float("inf")
    got = ctx.qk_norm_rope(q, k, norm=True)[0]
    assert bool(got[2, 1].isnan().all()) and bool(got[4, 0, 63].isnan()) and bool((got[4, 0, :63] == 0).all())
    got[2, 1], got[4, 0] = want[2, 1], want[4, 0]
    assert torch.equal(got, want)


@pytest.mark.parametrize("tokens", [2, 443, 444, 900, 3552, 3600])
def test_numbers_of_tokens_around_the_rules(ctx, tokens):
    """One token or up to eight per CTA, heads shared out over CTAs or not."""
    q, k, _ = _qkv(tokens, 6, 3, 128, torch.float16, tokens)
    pos, f = torch.arange(tokens).to(DEV), _freq(64)
    for x, got in zip((q, k), ctx.qk_norm_rope(q, k, pos, f)):
        want, bound = exact.rope(x, None, 1e-6, pos, f, False)
        exact.within(got, want, bound)


def test_refusals(ctx):
    from paper_2608_02611_b200.binding import KbError
    q, k, v = _qkv(4, 4, 2, 64, torch.bfloat16, 1)
    pos, f = torch.arange(4).to(DEV), _freq(32)
    cache = torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16, device=DEV)
    slots = torch.arange(4).to(DEV)
    bad = [
        dict(q=q.double()), dict(k=k[:3]), dict(k=k.float()), dict(q=q[:, :3]), dict(q=q.cpu()), dict(eps=0.0), dict(eps=float("nan")),
        dict(inv_freq=f.float()), dict(inv_freq=_freq(33)), dict(positions=pos.int()), dict(positions=pos[:3]), dict(positions=None),
        dict(q_weight=torch.ones(63, device=DEV)), dict(q_weight=torch.ones(64, device=DEV), k_weight=torch.ones(64, device=DEV).bfloat16()),
        dict(norm=False, q_weight=torch.ones(64, device=DEV)), dict(v=v), dict(slots=slots), dict(k_cache=cache, v=v, slots=slots),
        dict(k_cache=cache, v_cache=cache, v=v, slots=slots.int()), dict(k_cache=cache, v_cache=cache.half(), v=v, slots=slots),
        dict(k_cache=cache[:, :, :1], v_cache=cache[:, :, :1], v=v, slots=slots), dict(want_q=False, want_k=False),
        dict(q=q.transpose(0, 2)), dict(out=(q.float(), None)), dict(out=(q[:, :1].expand(4, 4, 64), None)), dict(out=(torch.empty(4, 4, 65, device=DEV, dtype=torch.bfloat16), None)),
        dict(q=q[:, :1].expand(4, 2 ** 32, 64)),
        dict(q=torch.zeros(4, 4, 257, device=DEV), k=torch.zeros(4, 2, 257, device=DEV), inv_freq=None),
    ]
    for change in bad:
        with pytest.raises((KbError, TypeError)):
            ctx.qk_norm_rope(**{**dict(q=q, k=k, positions=pos, inv_freq=f), **change})
    # no token: nothing to do
    qo, ko = ctx.qk_norm_rope(q[:0], k[:0], pos[:0], f)
    assert qo.shape == (0, 4, 64) and ko.shape == (0, 2, 64)
    assert ctx.poll() == 0
