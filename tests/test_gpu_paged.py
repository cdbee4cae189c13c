"""Attention of one new token over a paged cache, against 64 bits (bounds: attention_exact.py)."""
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


def _case(lens, hq, hkv, dim, dtype, page, seed, spare=3, fill=float("nan"), heads_first=False):
    """Queries and a cache whose slots past the lengths, and spare pages, hold `fill`; the same keys and values by sequence."""
    gen = _gen(seed)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=gen).to(torch.int32)
    table = torch.full((len(lens), max(1, max(need))), -5, dtype=torch.int32)
    kc, vc = (torch.full((pages, page, hkv, dim), fill, dtype=dtype) for _ in range(2))
    ks, vs, at = [], [], 0
    for s, n in enumerate(lens):
        table[s, :need[s]] = order[at:at + need[s]]
        at += need[s]
        k, v = (torch.randn(n, hkv, dim, generator=gen).to(dtype) for _ in range(2))
        for j in range(0, n, page):
            p, m = int(table[s, j // page]), min(page, n - j)
            kc[p, :m], vc[p, :m] = k[j:j + m], v[j:j + m]
        ks.append(k)
        vs.append(v)
    q = torch.randn(len(lens), hq, dim, generator=gen).to(dtype)
    if heads_first:
        kc, vc = (c.transpose(1, 2).contiguous().to(DEV).transpose(1, 2) for c in (kc, vc))
    return dict(q=q.to(DEV), k_cache=kc.to(DEV), v_cache=vc.to(DEV), table=table.to(DEV),
                lengths=torch.tensor(lens, dtype=torch.int32).to(DEV)), q, ks, vs


def _check(r, q, ks, vs, scale=None, what=""):
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    for s in range(q.shape[0]):
        seen = torch.ones(1, ks[s].shape[0], dtype=torch.bool)
        out, bound, lse, lse_bound = exact.attend(q[s:s + 1], ks[s], vs[s], seen, scale, q.dtype)
        exact.within(r.out[s:s + 1], out, bound, f"{what} sequence {s} of {ks[s].shape[0]} keys")
        if r.lse is not None:
            exact.within(r.lse[s:s + 1], lse, lse_bound, f"{what} lse of sequence {s}")


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("dim", [8, 40, 64, 72, 96, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (12, 12), (8, 1), (10, 2), (32, 4), (27, 3), (17, 1), (40, 1)])
def test_against_64_bits(ctx, dtype, dim, hq, hkv):
    """Groups of 1 to 40 query heads, lengths that end inside steps and pages, junk in every slot not seen."""
    lens = [1, 0, 15, 16, 17, 127, 128, 129, 300]
    kw, q, ks, vs = _case(lens, hq, hkv, dim, dtype, 16, dim * 100 + hq)
    _check(ctx.attention_paged(**kw, want_lse=True), q, ks, vs)


@pytest.mark.parametrize("page", [1, 5, 8, 16, 24, 48, 100, 128, 1024])
@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_pages_of_any_size_and_order(ctx, page, heads_first, dim):
    lens = [1, page, page + 1, 2 * page - 1 or 1, 333, 1000]
    kw, q, ks, vs = _case(lens, 8, 2, dim, torch.bfloat16, page, page, heads_first=heads_first)
    _check(ctx.attention_paged(**kw, want_lse=True), q, ks, vs)


@pytest.mark.parametrize("lens", [[5000], [9000, 3], [1, 20000], [0, 0, 7000, 0], [257] * 300 + [4000], [1] * 1000])
def test_long_and_many_sequences_divided_over_the_card(ctx, lens):
    kw, q, ks, vs = _case(lens, 4, 1, 128, torch.float16, 64, len(lens))
    r = ctx.attention_paged(**kw, want_lse=True)
    _check(r, q, ks, vs)
    again = ctx.attention_paged(**kw, want_lse=True)
    assert torch.equal(r.out, again.out) and torch.equal(r.lse, again.lse)       # the same order of every sum


def test_scores_that_rise_and_fall_and_extreme_ones(ctx):
    """Running references that have to be raised again and again; the largest score first, last, or everywhere."""
    for order in ("rising", "falling", "flat", "one"):
        kw, q, ks, vs = _case([2000], 2, 1, 64, torch.bfloat16, 16, 7)
        n = torch.arange(2000.0)
        gain = {"rising": n / 50, "falling": (2000 - n) / 50, "flat": torch.zeros(2000), "one": torch.where(n == 1234, 60.0, 0.0)}[order]
        k = (gain[:, None, None] * q[0, :1].float()).to(torch.bfloat16)
        table = kw["table"][0].cpu()
        for j in range(2000):
            kw["k_cache"][table[j // 16], j % 16] = k[j].to(DEV)
        _check(ctx.attention_paged(**kw, want_lse=True), q, [k], vs, what=order)


def test_scores_of_minus_infinity_and_nan(ctx):
    """A query all of whose scores are -infinity has zeros; NaN and +infinity reach their own heads, no others."""
    kw, q, ks, vs = _case([40, 40, 40], 2, 2, 64, torch.float16, 16, 3)
    kw["q"][0] = 0.0
    kw["q"][0, 0, 0] = 1.0
    kw["q"][1, 1, 3] = float("nan")
    t = kw["table"]
    for j in range(40):
        kw["k_cache"][t[0, j // 16], j % 16, 0, 0] = -math.inf
    r = ctx.attention_paged(**kw, want_lse=True)
    assert bool((r.out[0, 0] == 0).all()) and float(r.lse[0, 0]) == -math.inf
    assert bool(r.out[1, 1].isnan().all()) and bool(r.lse[1, 1].isnan())
    assert bool(r.out[0, 1].isfinite().all()) and bool(r.out[1, 0].isfinite().all()) and bool(r.out[2].isfinite().all())
    q2 = q.clone()
    _check(type(r)(r.out[2:], r.lse[2:]), q2[2:], ks[2:], vs[2:])
    kw["k_cache"][t[2, 1], 4, 1, 0] = math.inf
    kw["q"][2, 1, 0] = 1.0
    r = ctx.attention_paged(**kw, want_lse=True)
    assert bool(r.out[2, 1].isnan().all()) and bool(r.out[2, 0].isfinite().all())


def test_lengths_and_pages_that_are_not_there(ctx):
    """A page outside the cache, or a length beyond the table, is left out, touches nothing and shows in the status."""
    kw, q, ks, vs = _case([100, 100, 100, 100], 4, 2, 64, torch.bfloat16, 16, 5)
    good = ctx.attention_paged(**kw, want_lse=True)
    kw["table"][1, 2], kw["table"][2, 0], kw["lengths"][3] = 10 ** 6, -1, -7
    r = ctx.attention_paged(**kw, want_lse=True)
    assert ctx.poll() == 1 and ctx.poll() == 0
    assert torch.equal(r.out[0], good.out[0])
    part = [ks[1][torch.arange(100) // 16 != 2], ks[2][16:]], [vs[1][torch.arange(100) // 16 != 2], vs[2][16:]]
    _check(type(r)(r.out[1:3], r.lse[1:3]), q[1:3], *part)
    assert bool((r.out[3] == 0).all()) and bool((r.lse[3] == -math.inf).all())
    kw, q, ks, vs = _case([100], 4, 2, 64, torch.bfloat16, 16, 5)
    kw["lengths"][0] = 10 ** 9
    kw["table"] = kw["table"][:, :6]                                             # room for 96 keys
    r = ctx.attention_paged(**kw)
    assert ctx.poll() == 1 and ctx.poll() == 0
    _check(r, q, [ks[0][:96]], [vs[0][:96]])


def test_strided_queries_outputs_and_tables(ctx):
    kw, q, ks, vs = _case([50, 700], 8, 2, 64, torch.bfloat16, 16, 8)
    wide = torch.full((2, 12, 80), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, 2:10, 8:72] = kw["q"]
    kw["q"] = wide[:, 2:10, 8:72]
    held = torch.full((2, 60), 10 ** 8, dtype=torch.int32, device=DEV)
    held[:, 4:4 + kw["table"].shape[1]] = kw["table"]
    kw["table"] = held[:, 4:4 + kw["table"].shape[1]]
    for offset in (0, 1):                                       # outputs at any alignment
        out = torch.full((2 * 8 * 70 + 1,), 3.0, dtype=torch.bfloat16, device=DEV)
        view = out[offset:offset + 2 * 8 * 70].view(2, 8, 70)[..., :64]
        r = ctx.attention_paged(**kw, out=view)
        assert r.lse is None and r.out.data_ptr() == view.data_ptr()
        _check(r, q, ks, vs)
        assert bool((out[offset:offset + 2 * 8 * 70].view(2, 8, 70)[..., 64:] == 3.0).all())
    by_head = torch.zeros(8, 2, 64, dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    _check(ctx.attention_paged(**kw, out=by_head), q, ks, vs)


def test_scale(ctx):
    kw, q, ks, vs = _case([333], 4, 4, 64, torch.float16, 16, 2)
    for scale in (1.0, 1e-3, 2.5):
        _check(ctx.attention_paged(**kw, scale=scale, want_lse=True), q, ks, vs, scale)


def test_two_graphs_that_share_the_workspace_and_calls_between(ctx):
    """Counts that a launch leaves behind would show in the next one."""
    cases = [_case(lens, 8, 1, 128, torch.bfloat16, 32, i) for i, lens in enumerate([[9000, 1, 400], [30, 6000]])]
    want = [ctx.attention_paged(**c[0]).out for c in cases]
    graphs, outs = [], []
    for c in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(ctx.attention_paged(**c[0]).out)
        graphs.append(g)
    for _ in range(3):
        for i in (0, 1):
            outs[i].zero_()
            graphs[i].replay()
            assert torch.equal(outs[i], want[i])
            assert torch.equal(ctx.attention_paged(**cases[1 - i][0]).out, want[1 - i])


def test_a_first_call_inside_a_capture_is_refused_unless_reserved():
    from paper_2608_02611_b200 import binding
    kw, q, ks, vs = _case([100], 2, 2, 64, torch.float16, 16, 1)
    for reserve in (False, True):
        c = binding.Context(0)
        if reserve:
            c.reserve_attention_paged()
        g = torch.cuda.CUDAGraph()
        out = torch.zeros(1, 2, 64, dtype=torch.float16, device=DEV)
        with torch.cuda.graph(g):
            if reserve:
                c.attention_paged(**kw, out=out)
            else:
                with pytest.raises(binding.KbError, match="KB_ERR_WORKSPACE"):
                    c.attention_paged(**kw, out=out)
                out.add_(0)
        g.replay()
        if reserve:
            _check(binding.AttentionResult(out, None), q, ks, vs)
        assert c.poll() == 0
        c.close()


@pytest.mark.parametrize("n", [1, 18, 19, 36, 37, 74, 256, 257, 600])
def test_numbers_of_sequences_around_the_rules(ctx, n):
    """Eight warps or four, up to a CTA's threads of sequences or more, pieces that begin and end inside sequences."""
    lens = [(53 * i) % 310 for i in range(n)]
    lens[0] = 777
    kw, q, ks, vs = _case(lens, 8, 8, 64, torch.bfloat16, 16, n)
    _check(ctx.attention_paged(**kw, want_lse=True), q, ks, vs)


@pytest.mark.parametrize("hkv", [1, 9, 20, 40, 100, 200, 500])
def test_numbers_of_groups_that_do_not_divide_the_card(ctx, hkv):
    kw, q, ks, vs = _case([300, 40, 0, 1000], hkv, hkv, 16, torch.float16, 16, hkv)
    _check(ctx.attention_paged(**kw, want_lse=True), q, ks, vs)


def test_two_contexts_on_two_streams_at_once():
    """Each has its own parts and counts."""
    from paper_2608_02611_b200 import binding
    cases = [_case(lens, 8, 1, 128, torch.bfloat16, 32, i) for i, lens in enumerate([[9000, 1, 400], [30, 6000]])]
    contexts = [binding.Context(0) for _ in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [[], []]
    torch.cuda.synchronize()
    for _ in range(5):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                outs[i].append(contexts[i].attention_paged(**cases[i][0], want_lse=True))
    torch.cuda.synchronize()
    for i in (0, 1):
        _check(outs[i][0], *cases[i][1:])
        for r in outs[i][1:]:
            assert torch.equal(r.out, outs[i][0].out)
        assert contexts[i].poll() == 0
        contexts[i].close()


def test_refusals(ctx):
    from paper_2608_02611_b200.binding import KbError
    kw, *_ = _case([20, 20], 4, 2, 64, torch.float16, 16, 1)
    bad = [
        dict(q=kw["q"].float()), dict(q=kw["q"].bfloat16()), dict(q=kw["q"][:, :3]), dict(q=kw["q"][:1]), dict(q=kw["q"].cpu()),
        dict(q=kw["q"][..., :60]), dict(k_cache=kw["k_cache"].bfloat16()), dict(k_cache=kw["k_cache"][:, :8]), dict(k_cache=kw["k_cache"][:, :, :1]),
        dict(table=kw["table"].long()), dict(table=kw["table"][:1]), dict(table=kw["table"][0]), dict(lengths=kw["lengths"].long()),
        dict(lengths=kw["lengths"][:1]), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=3e38), dict(scale=float("nan")),
        dict(out=kw["q"].float()), dict(out=kw["q"][:, :2]), dict(out=kw["q"][:, :1].expand(2, 4, 64)),
        dict(q=torch.zeros(2 * 4 * 64 + 1, dtype=torch.float16, device=DEV)[1:].view(2, 4, 64)),          # not on 16 bytes
        dict(q=torch.zeros(2, 4, 136, dtype=torch.float16, device=DEV), k_cache=torch.zeros(2, 16, 2, 136, dtype=torch.float16, device=DEV),
             v_cache=torch.zeros(2, 16, 2, 136, dtype=torch.float16, device=DEV)),
    ]
    for change in bad:
        with pytest.raises((KbError, TypeError)):
            ctx.attention_paged(**{**kw, **change})
    r = ctx.attention_paged(kw["q"][:0], kw["k_cache"], kw["v_cache"], kw["table"][:0], kw["lengths"][:0], want_lse=True)
    assert r.out.shape == (0, 4, 64) and r.lse.shape == (0, 4)
    # a cache without pages, for empty sequences only
    r = ctx.attention_paged(kw["q"], kw["k_cache"][:0], kw["v_cache"][:0], kw["table"][:, :0], kw["lengths"] * 0)
    assert bool((r.out == 0).all())
    assert ctx.poll() == 0
