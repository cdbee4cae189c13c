"""Attention over packed prompts, against 64 bits (bounds: attention_exact.py)."""
import math

import pytest
import torch

from tests import attention_exact as exact

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
    return torch.tensor([0] + list(lens)).cumsum(0).to(torch.int32)


def _inputs(nq, nk, hq, hkv, dim, dtype, seed):
    gen = _gen(seed)
    return [torch.randn(n, h, dim, generator=gen).to(dtype) for n, h in ((nq, hq), (nk, hkv), (nk, hkv))]


def _seen(nq, nk, causal):
    return torch.arange(nk) <= (torch.arange(nq)[:, None] + nk - nq if causal else torch.full((nq, 1), nk))


def _check(r, q, k, v, qlens, klens, causal, scale=None, rows=None):
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    qa = ka = 0
    for s, (nq, nk) in enumerate(zip(qlens, klens)):
        seen = _seen(nq, nk, causal)
        pick = torch.arange(nq) if rows is None else torch.arange(nq)[rows(nq)]
        out, bound, lse, lse_bound = exact.attend(q[qa:qa + nq][pick], k[ka:ka + nk], v[ka:ka + nk], seen[pick], scale, q.dtype)
        exact.within(r.out[qa:qa + nq].cpu()[pick], out, bound, f"sequence {s}: {nq} x {nk}")
        if r.lse is not None:
            exact.within(r.lse[qa:qa + nq].cpu()[pick], lse, lse_bound, f"lse of sequence {s}")
        qa, ka = qa + nq, ka + nk


# lengths that end inside and at tiles of 128 and pieces of 256 queries, empty sequences among them
LENS = [[1], [128], [129], [256, 1], [77, 0, 128, 300, 3], [257, 511, 2, 640]]


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("hq,hkv,dim", [(2, 1, 128), (3, 3, 64), (4, 2, 64), (5, 1, 128)])
def test_against_64_bits(ctx, lens, causal, dtype, hq, hkv, dim):
    q, k, v = _inputs(sum(lens), sum(lens), hq, hkv, dim, dtype, sum(lens) + dim)
    r = ctx.attention(q.to(DEV), k.to(DEV), v.to(DEV), _offsets(lens).to(DEV), causal=causal, want_lse=True)
    assert r.out.dtype == dtype and r.lse.dtype == torch.float32
    _check(r, q, k, v, lens, lens, causal)


@pytest.mark.parametrize("dim", [8, 16, 40, 72, 80, 96, 120])
def test_dims(ctx, dim):
    for dtype in HALVES:
        q, k, v = _inputs(200, 200, 4, 2, dim, dtype, dim)
        _check(ctx.attention(q.to(DEV), k.to(DEV), v.to(DEV), want_lse=True), q, k, v, [200], [200], True)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (16, 1), (7, 1), (12, 4)])
def test_groups(ctx, hq, hkv):
    lens = [130, 400]
    q, k, v = _inputs(530, 530, hq, hkv, 64, torch.bfloat16, hq)
    _check(ctx.attention(q.to(DEV), k.to(DEV), v.to(DEV), _offsets(lens).to(DEV), want_lse=True), q, k, v, lens, lens, True)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("group", [1, 2])
def test_other_numbers_of_keys_than_queries(ctx, causal, group):
    """Queries at the end of longer texts; more queries than keys, the first of which see nothing; no queries, no keys."""
    qlens, klens = [1, 100, 300, 256, 200, 0, 50, 400], [700, 260, 301, 128, 70, 33, 0, 1]
    q, k, v = _inputs(sum(qlens), sum(klens), 2 * group, 2, 64, torch.bfloat16, 5)
    r = ctx.attention(q.to(DEV), k.to(DEV), v.to(DEV), _offsets(qlens).to(DEV), _offsets(klens).to(DEV), causal=causal, want_lse=True)
    _check(r, q, k, v, qlens, klens, causal)
    assert bool((r.out[-450:-400] == 0).all()) and bool((r.lse[-450:-400] == -math.inf).all())


def test_no_key_at_all(ctx):
    q, k, v = _inputs(5, 0, 2, 2, 64, torch.float16, 1)
    r = ctx.attention(q.to(DEV), k.to(DEV), v.to(DEV), _offsets([5]).to(DEV), _offsets([0]).to(DEV), want_lse=True)
    assert bool((r.out == 0).all()) and bool((r.lse == -math.inf).all())


@pytest.mark.parametrize("dtype", HALVES)
def test_long_prompts(ctx, dtype):
    """Some rows of prompts of many tiles."""
    lens = [5000, 2300]
    q, k, v = _inputs(7300, 7300, 2, 1, 128, dtype, 3)
    r = ctx.attention(q.to(DEV), k.to(DEV), v.to(DEV), _offsets(lens).to(DEV), want_lse=True)
    _check(r, q, k, v, lens, lens, True, rows=lambda n: torch.arange(0, n, 37) if n else [])
    again = ctx.attention(q.to(DEV), k.to(DEV), v.to(DEV), _offsets(lens).to(DEV), want_lse=True)
    assert torch.equal(r.out, again.out) and torch.equal(r.lse, again.lse)


def test_many_sequences(ctx):
    lens = [(7 * i) % 40 for i in range(900)]
    q, k, v = _inputs(sum(lens), sum(lens), 2, 2, 64, torch.float16, 4)
    r = ctx.attention(q.to(DEV), k.to(DEV), v.to(DEV), _offsets(lens).to(DEV), want_lse=True)
    _check(r, q, k, v, lens, lens, True)


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("group", [1, 2, 3])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens", LENS + [[1], [900], [40] * 40])
def test_heads_many_and_few_give_the_same_bits(ctx, lens, dim, group, dtype):
    """Calls with few items take one tile at a time, others two heads or two pieces: no output shows which.  Values that
    are not finite lie behind what some queries see."""
    q, k, v = (t.to(DEV) for t in _inputs(sum(lens), sum(lens), group, 1, dim, dtype, 8))
    v[-1, :, :3] = float("nan")
    v[sum(lens) // 2, :, 5] = float("inf")
    offsets, heads = _offsets(lens).to(DEV), 300 // group
    many = [t.repeat(1, heads, 1) for t in (q, k, v)]
    for causal in (True, False):
        few, all_ = ctx.attention(q, k, v, offsets, causal=causal, want_lse=True), ctx.attention(*many, offsets, causal=causal, want_lse=True)
        assert torch.equal(few.out.repeat(1, heads, 1).view(torch.int16), all_.out.view(torch.int16))
        assert torch.equal(few.lse.repeat(1, heads).view(torch.int32), all_.lse.view(torch.int32))
    assert ctx.poll() == 0


@pytest.mark.parametrize("hq,hkv", [(32, 32), (32, 16)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", [
    [300, 2100, 0, 1, 1500, 2100, 129, 4000, 64, 777],
    [16, 5000, 8000],
    [9000],
    [340] * 29 + [0, 1, 300],
])
def test_more_keys_than_the_cache_holds(ctx, lens, causal, hq, hkv):
    """Then sequences are worked on in phases, whose order no output shows: each is what a call of its own gives, and some
    rows are compared with 64 bits."""
    tokens = sum(lens)
    assert 4 * tokens * hkv * 128 > 64 << 20
    q, k, v = (t.to(DEV) for t in _inputs(tokens, tokens, hq, hkv, 128, torch.bfloat16, 5))
    offsets = _offsets(lens).to(DEV)
    out = torch.full_like(q, float("nan"))
    r = ctx.attention(q, k, v, offsets, causal=causal, want_lse=True, out=out)
    at = 0
    for n in lens:
        if n:
            one = ctx.attention(q[at:at + n], k[at:at + n], v[at:at + n], causal=causal, want_lse=True)
            assert torch.equal(one.out, out[at:at + n]) and torch.equal(one.lse, r.lse[at:at + n]), (at, n)
        at += n
    assert ctx.poll() == 0
    _check(r, q.cpu(), k.cpu(), v.cpu(), lens, lens, causal, rows=lambda n: [0, n // 2, n - 1] if n else [])


@pytest.mark.parametrize("order", ["rising", "falling", "steps"])
def test_scores_that_rise_and_fall(ctx, order):
    """References that have to be raised tile after tile, by small and by huge amounts."""
    n = 900
    q, k, v = _inputs(n, n, 2, 1, 64, torch.bfloat16, 6)
    q[:] = q[:1, :1]
    j = torch.arange(float(n))
    gain = {"rising": j / 40, "falling": (n - j) / 40, "steps": (j // 128) * 3.0}[order]
    k = (gain[:, None, None] * q[0, :1].float()).to(torch.bfloat16)
    for causal in (True, False):
        r = ctx.attention(q.to(DEV), k.to(DEV), v.to(DEV), causal=causal, want_lse=True)
        _check(r, q, k, v, [n], [n], causal)


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("group", [1, 2])
def test_what_a_query_does_not_see_does_not_touch_it(ctx, dtype, group):
    """NaN and infinities in keys and values of later tokens, of other sequences and behind the last one."""
    lens = [100, 200, 333]
    n = sum(lens)
    q, k, v = _inputs(n + 40, n + 40, 2 * group, 2, 64, dtype, 8)
    q[n:], k[n:], v[n:] = math.nan, math.inf, math.nan
    bad = {99: math.nan, 250: math.inf, 299: -math.inf, 500: math.nan, 632: math.inf}       # tokens whose values are broken
    for t, x in bad.items():
        v[t, 0, 5] = x
        k[t, 1, 3] = x
    out = torch.full((n + 40, 2 * group, 64), 9.0, dtype=dtype, device=DEV)
    r = ctx.attention(q.to(DEV), k.to(DEV), v.to(DEV), _offsets(lens).to(DEV), want_lse=True, out=out)
    assert bool((r.out[n:] == 9.0).all())
    a = 0
    for m in lens:
        rows = torch.arange(m)
        first = min([t - a for t in bad if a <= t < a + m])
        clean = rows < first                         # rows that see none of the broken tokens
        part = [x[a:a + m] for x in (q, k, v)]
        zero = [torch.where(x.isfinite(), x, torch.zeros_like(x)) for x in part[1:]]
        want, bound, lse, lse_bound = exact.attend(part[0], *zero, _seen(m, m, True), 0.125, dtype)
        got, got_lse = r.out[a:a + m].cpu(), r.lse[a:a + m].cpu()
        exact.within(got[clean], want[clean], bound[clean])
        exact.within(got_lse[clean], lse[clean], lse_bound[clean])
        # broken values reach their own element of their own heads, and only there
        first_heads = got[:, :group].double()
        assert bool((~first_heads[~clean][..., 5].isfinite()).all())
        first_heads[..., 5] = want[:, :group, 5]
        exact.within(first_heads, want[:, :group], bound[:, :group])
        a += m


def test_non_finite_queries_keys_and_scores(ctx):
    q, k, v = _inputs(300, 300, 2, 2, 64, torch.bfloat16, 2)
    q[10, 0, 0] = math.nan
    q[20, 1], k[:, 1, 0] = 0.0, torch.where(torch.arange(300) < 50, -math.inf, 0.0)
    q[20, 1, 0] = 1.0                                   # all scores of query 20 are -infinity
    q[30, 0, 0], k[7, 0, 0] = 1.0, math.inf             # a score of +infinity
    q[:, 1, 0] = q[:, 1, 0].abs()
    r = ctx.attention(q.to(DEV), k.to(DEV), v.to(DEV), want_lse=True)
    assert bool(r.out[10, 0].isnan().all()) and bool(r.lse[10, 0].isnan()) and bool(r.out[10, 1].isfinite().all())
    assert bool((r.out[20, 1] == 0).all()) and float(r.lse[20, 1]) == -math.inf
    assert bool(r.out[30, 0].isnan().all())
    assert bool(r.out[:7, 0].isfinite().all())


def test_slices_of_one_projection_and_any_output(ctx):
    """Strided heads; heads first; outputs that are not 16-byte aligned; gaps that stay as they were."""
    n, hq, hkv, dim = 150, 4, 2, 64
    qkv = torch.randn(n, hq + 2 * hkv, dim, generator=_gen(1)).to(torch.bfloat16)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    d = qkv.to(DEV)
    views = [(d[:, :hq], d[:, hq:hq + hkv], d[:, hq + hkv:])]
    t = d.transpose(0, 1).contiguous().transpose(0, 1)
    views.append((t[:, :hq], t[:, hq:hq + hkv], t[:, hq + hkv:]))
    for a, b, c in views:
        _check(ctx.attention(a, b, c, want_lse=True), q, k, v, [n], [n], True)
        for offset in (0, 1):
            held = torch.full((n * hq * 70 + 1,), 5.0, dtype=torch.bfloat16, device=DEV)
            view = held[offset:offset + n * hq * 70].view(n, hq, 70)
            _check(ctx.attention(a, b, c, out=view[..., :64]), q, k, v, [n], [n], True)
            assert bool((view[..., 64:] == 5.0).all())
        heads_first = torch.zeros(hq, n, dim, dtype=torch.bfloat16, device=DEV).transpose(0, 1)
        _check(ctx.attention(a, b, c, out=heads_first), q, k, v, [n], [n], True)


def test_scale(ctx):
    q, k, v = _inputs(140, 140, 2, 2, 64, torch.float16, 9)
    for scale in (1.0, 1e-4, 3.0):
        _check(ctx.attention(q.to(DEV), k.to(DEV), v.to(DEV), scale=scale, want_lse=True), q, k, v, [140], [140], True, scale)


@pytest.mark.parametrize("offsets", [[0, 50, 40, 100], [-3, 50, 100, 100], [0, 50, 100, 101], [5, 60, 80, 99]])
def test_offsets_that_are_wrong_show_and_touch_nothing(ctx, offsets):
    """Sequences whose offsets are out of range or descend are left out; the last list is right and leaves rows out."""
    q, k, v = _inputs(100, 100, 2, 1, 64, torch.bfloat16, 7)
    out = torch.full((100, 2, 64), 4.0, dtype=torch.bfloat16, device=DEV)
    ctx.attention(q.to(DEV), k.to(DEV), v.to(DEV), torch.tensor(offsets, dtype=torch.int32).to(DEV), out=out)
    right = offsets[0] == 5
    assert ctx.poll() == (0 if right else 1) and ctx.poll() == 0
    if right:
        assert bool((out[:5] == 4.0).all()) and bool((out[99:] == 4.0).all())
        for a, b in ((5, 60), (60, 80), (80, 99)):
            r = ctx.attention(q[a:b].to(DEV), k[a:b].to(DEV), v[a:b].to(DEV))
            assert torch.equal(out[a:b], r.out)


def test_in_graphs_with_new_lengths(ctx):
    """A captured call takes its lengths at each replay."""
    q, k, v = _inputs(600, 600, 4, 2, 128, torch.bfloat16, 7)
    d = [x.to(DEV) for x in (q, k, v)]
    offsets = _offsets([300, 300]).to(DEV)
    ctx.attention(*d, offsets)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r = ctx.attention(*d, offsets, want_lse=True)
    for lens in ([300, 300], [1, 599], [600, 0], [129, 471]):
        offsets.copy_(_offsets(lens))
        g.replay()
        _check(r, q, k, v, lens, lens, True, rows=lambda n: torch.arange(0, n, 11) if n else [])


def test_a_first_call_inside_a_capture_and_on_another_stream():
    from paper_2608_02611_b200 import binding
    c = binding.Context(0)
    q, k, v = _inputs(200, 200, 4, 2, 64, torch.float16, 3)
    d = [x.to(DEV) for x in (q, k, v)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r = c.attention(*d, want_lse=True)
    g.replay()
    _check(r, q, k, v, [200], [200], True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s = c.attention(*d, want_lse=True)
    side.synchronize()
    assert torch.equal(s.out, r.out) and torch.equal(s.lse, r.lse)
    assert c.poll() == 0
    c.close()


def test_two_contexts_on_two_streams_at_once():
    """Each has its count of items; calls of one take turns on the card with the other's, products of another kernel with
    tensor memory among them."""
    from paper_2608_02611_b200 import binding
    lens = [900, 3, 400, 0, 257]
    q, k, v = (t.to(DEV) for t in _inputs(sum(lens), sum(lens), 40, 8, 128, torch.bfloat16, 9))
    offsets = _offsets(lens).to(DEV)
    both = [(binding.Context(0), torch.cuda.Stream()) for _ in range(2)]
    want = both[0][0].attention(q, k, v, offsets, want_lse=True)
    x, s = both[0][0].quantize_blocks(q.reshape(sum(lens), -1))
    w, ws = both[0][0].quantize_blocks(torch.randn(512, x.shape[1], device=DEV), tiles=True)
    product = both[0][0].matmul_blocks(x, s, w, ws)
    torch.cuda.synchronize()
    got = []
    for _ in range(40):
        for ctx, stream in both:
            with torch.cuda.stream(stream):
                got.append((ctx.attention(q, k, v, offsets, want_lse=True), ctx.matmul_blocks(x, s, w, ws)))
    torch.cuda.synchronize()
    for r, p in got:
        assert torch.equal(r.out, want.out) and torch.equal(r.lse, want.lse) and torch.equal(p, product)
    for ctx, _ in both:
        assert ctx.poll() == 0
        ctx.close()


def test_no_gradient_and_any_rank_of_inputs_that_require_one(ctx):
    q, k, v = (x.to(DEV).requires_grad_(True) for x in _inputs(20, 20, 2, 1, 64, torch.bfloat16, 3))
    r = ctx.attention(q, k, v, want_lse=True)
    assert not r.out.requires_grad and not r.lse.requires_grad
    a, b = ctx.qk_norm_rope(q, k)
    assert not a.requires_grad and not b.requires_grad


@pytest.mark.parametrize("n", [1, 31, 32, 33, 64, 65])
def test_numbers_of_sequences_around_a_warps(ctx, n):
    """Up to 32 sequences are handed out by length, more of them one after the other."""
    lens = [(37 * i) % 300 for i in range(n)]
    lens[-1] = 260
    klens = [m + (11 * i) % 90 for i, m in enumerate(lens)]
    q, k, v = _inputs(sum(lens), sum(klens), 2, 2, 64, torch.bfloat16, n)
    for causal in (True, False):
        r = ctx.attention(q.to(DEV), k.to(DEV), v.to(DEV), _offsets(lens).to(DEV), _offsets(klens).to(DEV), causal=causal, want_lse=True)
        _check(r, q, k, v, lens, klens, causal, rows=lambda m: torch.arange(0, m, 3) if m else [])


def test_refusals(ctx):
    from paper_2608_02611_b200.binding import KbError
    q, k, v = (x.to(DEV) for x in _inputs(20, 20, 4, 2, 64, torch.float16, 1))
    o = _offsets([20]).to(DEV)
    wide = torch.zeros(20, 4, 136, dtype=torch.float16, device=DEV)
    odd = torch.zeros(20 * 4 * 64 + 1, dtype=torch.float16, device=DEV)[1:].view(20, 4, 64)
    bad = [
        dict(q=q.float(), k=k.float(), v=v.float()), dict(q=q.bfloat16()), dict(q=q[:, :3]), dict(q=q.cpu()), dict(q=odd), dict(q=wide, k=wide, v=wide),
        dict(q=q[..., :60], k=k[..., :60], v=v[..., :60]), dict(v=v[:, :1]), dict(v=v[:10]), dict(k=k[:10], v=v[:10]), dict(k=k[..., :56]),
        dict(q_offsets=o.long()), dict(q_offsets=o[:0]), dict(q_offsets=None, k_offsets=o), dict(k_offsets=_offsets([10, 10]).to(DEV)),
        dict(scale=0.0), dict(scale=float("nan")), dict(scale=-2.0), dict(scale=3e38), dict(out=q.float()), dict(out=q[:, :2]), dict(out=q[:1].expand(20, 4, 64)),
        dict(k=k[:, :1].expand(20, 2, 64)), dict(q=q.transpose(0, 2)), dict(q=q[0]),
    ]
    for change in bad:
        with pytest.raises((KbError, TypeError)):
            ctx.attention(**{**dict(q=q, k=k, v=v, q_offsets=o), **change})
    r = ctx.attention(q[:0], k, v, _offsets([0]).to(DEV), o, want_lse=True)
    assert r.out.shape == (0, 4, 64) and r.lse.shape == (0, 4)
    r = ctx.attention(q, k, v, o[:1])                       # no sequence: nothing is written
    assert r.out.shape == q.shape
    assert ctx.poll() == 0


def test_a_prompt_then_tokens_as_a_server_makes_them(ctx):
    """Norm and rotation store a prompt's keys, its attention runs, new tokens follow one by one from the cache: the same
    numbers as the whole text at once."""
    hq, hkv, dim, page, dtype = 8, 2, 64, 16, torch.bfloat16
    lens, new = [45, 130], 3
    gen = _gen(12)
    total = [n + new for n in lens]
    x = [torch.randn(n, hq + 2 * hkv, dim, generator=gen).to(dtype).to(DEV) for n in total]
    f = (1e4 ** (-torch.arange(32, dtype=torch.float64) / 32)).to(DEV)
    wq, wk = (torch.rand(dim, generator=gen).add(0.5).to(dtype).to(DEV) for _ in range(2))
    cut = lambda t: (t[:, :hq], t[:, hq:hq + hkv], t[:, hq + hkv:])   # noqa: E731
    # the whole texts at once
    whole = torch.cat(x)
    positions = torch.cat([torch.arange(n) for n in total]).to(DEV)
    q, k, v = cut(whole)
    q, k = ctx.qk_norm_rope(q, k, positions, f, wq, wk)
    want = ctx.attention(q, k, v, _offsets(total).to(DEV))
    # prompts, then tokens
    pages = 20
    kc, vc = (torch.full((pages, page, hkv, dim), math.nan, dtype=dtype, device=DEV) for _ in range(2))
    table = torch.randperm(pages, generator=gen)[:18].view(2, 9).to(torch.int32).to(DEV)
    slot = lambda s, at: table[s, at // page].long() * page + at % page   # noqa: E731
    prompt = torch.cat([t[:n] for t, n in zip(x, lens)])
    at = [torch.arange(n, device=DEV) for n in lens]
    q, k, v = cut(prompt)
    slots = torch.cat([slot(s, at[s]) for s in (0, 1)])
    q, k = ctx.qk_norm_rope(q, k, torch.cat(at), f, wq, wk, v=v, k_cache=kc, v_cache=vc, slots=slots)
    got = ctx.attention(q, k, v, _offsets(lens).to(DEV))
    starts = [0, total[0]]
    assert torch.equal(got.out[:lens[0]], want.out[:lens[0]]) and torch.equal(got.out[lens[0]:], want.out[total[0]:total[0] + lens[1]])
    for i in range(new):
        step = torch.stack([x[s][lens[s] + i] for s in (0, 1)])
        pos = torch.tensor([n + i for n in lens], device=DEV)
        q, k, v = cut(step)
        q, _ = ctx.qk_norm_rope(q, k, pos, f, wq, wk, want_k=False, v=v, k_cache=kc, v_cache=vc,
                                slots=torch.stack([slot(s, pos[s]) for s in (0, 1)]))
        r = ctx.attention_paged(q, kc, vc, table, (pos + 1).to(torch.int32))
        for s in (0, 1):
            w = want.out[starts[s] + lens[s] + i].double()
            # two ways of rounding p and the result: 2 half steps each, of values of at most the largest |v|
            assert float((r.out[s].double() - w).abs().max()) <= 4 * 2.0 ** -8 * float(whole[:, hq + hkv:].abs().max())
