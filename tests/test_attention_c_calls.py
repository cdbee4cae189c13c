"""The attention operators' C entry points, called through ctypes as a program without torch's binding calls them."""
import ctypes

import pytest
import torch

F32, F16, BF16 = 0, 1, 2


def test_a_null_context_is_refused_without_a_device():
    from paper_2608_02611_b200 import binding
    L = binding.load()
    cache = binding.PagedCache(None, None, 8, 8, 8, 8, 8, 8, 1, 16)
    assert L.kb_qk_norm_rope(None, None, 8, 8, 1, None, 8, 8, 1, 1, 8, BF16, 0, None, None, BF16, 0.0, None, None, 0, 0, None, 8, 8, None, 8, 8,
                             None, 8, 8, ctypes.byref(cache), None, None) == 1
    assert L.kb_attention(None, None, 8, 8, 1, 1, None, 8, 8, None, 8, 8, 1, 1, 8, BF16, None, None, 1, 1, 1.0, None, 8, 8, None, None) == 1
    assert L.kb_attention_paged(None, None, 8, 8, 1, ctypes.byref(cache), 1, 8, BF16, None, 0, 0, None, 1, 1.0, None, 8, 8, None, None) == 1
    assert L.kb_attention_paged_reserve(None, None) == 1


@pytest.fixture(scope="module")
def ctx():
    from paper_2608_02611_b200 import binding
    c = binding.Context(0)
    yield c
    assert c.poll() == 0
    c.close()


@pytest.mark.gpu
def test_the_three_calls_make_what_the_python_calls_make(ctx):
    """A prompt of 70 tokens to a cache of pages of 16, and its last token once more from there."""
    from paper_2608_02611_b200 import binding
    L = binding.load()
    n, hq, hkv, dim, page, pages = 70, 6, 2, 64, 16, 8
    gen = torch.Generator()
    gen.manual_seed(1)
    x = torch.randn(n, hq + 2 * hkv, dim, generator=gen).bfloat16().cuda()
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    pos = torch.arange(n, device="cuda")
    freq = 1e4 ** (-torch.arange(dim // 2, dtype=torch.float64, device="cuda") / (dim // 2))
    table = torch.randperm(pages, generator=gen).to(torch.int32).cuda().view(1, pages)
    slots = table[0, pos // page].long() * page + pos % page
    length = torch.tensor([n], dtype=torch.int32, device="cuda")

    def storage():
        return [torch.zeros(pages, page, hkv, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    kc, vc = storage()
    want_q, want_k = ctx.qk_norm_rope(q, k, pos, freq, v=v, k_cache=kc, v_cache=vc, slots=slots)
    want = ctx.attention(want_q, want_k, v, want_lse=True)
    want_last = ctx.attention_paged(want_q[-1:], kc, vc, table, length, want_lse=True)

    st = torch.cuda.current_stream().cuda_stream
    row = (hq + 2 * hkv) * dim
    kc2, vc2 = storage()
    cache = binding.PagedCache(kc2.data_ptr(), vc2.data_ptr(), page * hkv * dim, hkv * dim, dim, page * hkv * dim, hkv * dim, dim, pages, page)
    got_q, got_k, out = torch.empty_like(want_q), torch.empty_like(want_k), torch.empty_like(want.out)
    lse = torch.empty_like(want.lse)
    assert L.kb_qk_norm_rope(ctx._h, q.data_ptr(), row, dim, hq, k.data_ptr(), row, dim, hkv, n, dim, BF16, 1, None, None, BF16, 1e-6, pos.data_ptr(),
                             freq.data_ptr(), dim, 0, got_q.data_ptr(), hq * dim, dim, got_k.data_ptr(), hkv * dim, dim, v.data_ptr(), row, dim,
                             ctypes.byref(cache), slots.data_ptr(), st) == 0
    assert L.kb_attention(ctx._h, got_q.data_ptr(), hq * dim, dim, hq, n, got_k.data_ptr(), hkv * dim, dim, v.data_ptr(), row, dim, hkv, n, dim, BF16,
                          None, None, 1, 1, dim ** -0.5, out.data_ptr(), hq * dim, dim, lse.data_ptr(), st) == 0
    assert torch.equal(got_q, want_q) and torch.equal(got_k, want_k) and torch.equal(kc2, kc) and torch.equal(vc2, vc)
    assert torch.equal(out, want.out) and torch.equal(lse, want.lse)
    last, last_lse = torch.empty_like(want_last.out), torch.empty_like(want_last.lse)
    assert L.kb_attention_paged_reserve(ctx._h, st) == 0
    assert L.kb_attention_paged(ctx._h, got_q[-1:].data_ptr(), hq * dim, dim, hq, ctypes.byref(cache), hkv, dim, BF16, table.data_ptr(), pages, pages,
                                length.data_ptr(), 1, dim ** -0.5, last.data_ptr(), hq * dim, dim, last_lse.data_ptr(), st) == 0
    assert torch.equal(last, want_last.out) and torch.equal(last_lse, want_last.lse)


@pytest.mark.gpu
def test_what_only_a_c_call_can_ask_for_is_refused(ctx):
    from paper_2608_02611_b200 import binding
    L = binding.load()
    x = torch.zeros(64 * 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(x, 3.0)
    number = torch.zeros(8, dtype=torch.int64, device="cuda")
    p, o, i = x.data_ptr(), out.data_ptr(), number.data_ptr()

    def paged(**change):
        a = dict(q=p, q_row=64, q_head=64, q_heads=1, cache=binding.PagedCache(p, p, 1024, 64, 64, 1024, 64, 64, 1, 16), hkv=1, dim=64, dtype=BF16, table=i,
                 table_row=1, max_pages=1, lengths=i, sequences=1, scale=1.0, out=o, o_row=64, o_head=64, lse=None, stream=None)
        a.update(change)
        a["cache"] = ctypes.byref(a["cache"]) if a["cache"] else None
        return L.kb_attention_paged(ctx._h, *a.values())

    def prompt(**change):
        a = dict(q=p, q_row=64, q_head=64, q_heads=1, q_tokens=4, k=p, k_row=64, k_head=64, v=p, v_row=64, v_head=64, hkv=1, k_tokens=4, dim=64, dtype=BF16,
                 q_offsets=None, k_offsets=None, sequences=1, causal=1, scale=1.0, out=o, o_row=64, o_head=64, lse=None, stream=None)
        return L.kb_attention(ctx._h, *{**a, **change}.values())

    held = binding.PagedCache
    for change in (dict(cache=None), dict(lengths=None), dict(table=None), dict(lengths=i + 2), dict(table=i + 1), dict(q=None), dict(out=None), dict(q=p + 2),
                   dict(cache=held(None, p, 1024, 64, 64, 1024, 64, 64, 1, 16)), dict(cache=held(p, p, 1024, 64, 64, 1024, 64, 64, 1, 0)),
                   dict(cache=held(p, p, 1024, 60, 64, 1024, 64, 64, 1, 16)), dict(cache=held(p, p, 1024, 0, 64, 1024, 64, 64, 1, 16)),
                   dict(cache=held(p, p, 1024, 64, 64, 1024, 64, 64, 1 << 31, 16)), dict(max_pages=1 << 28), dict(dim=0), dict(dim=68), dict(dim=136),
                   dict(dtype=F32), dict(q_heads=0), dict(hkv=0), dict(q_heads=3, hkv=2), dict(scale=0.0), dict(scale=float("inf")), dict(sequences=2, table_row=0)):
        assert paged(**change) in (1, 2, 3), change
    for change in (dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q_offsets=i), dict(k_offsets=i), dict(sequences=2), dict(sequences=0), dict(causal=2),
                   dict(q_row=60), dict(k_row=0), dict(v=p + 8), dict(lse=o + 2), dict(o_row=63), dict(q_offsets=i + 1, k_offsets=i), dict(dim=12), dict(scale=-1.0),
                   dict(k_tokens=(1 << 24) + 1), dict(q_tokens=(1 << 30) + 1), dict(dtype=F32), dict(q_row=1 << 39)):
        assert prompt(**change) in (1, 2, 3), change
    assert bool((out == 3.0).all())
    assert paged(sequences=0) == 0 and prompt(q_tokens=0) == 0 and ctx.poll() == 0
