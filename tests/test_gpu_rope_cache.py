"""What the rotation takes as a cache to write to."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
PAGES, PAGE, HEADS, DIM = 3, 16, 2, 64


@pytest.fixture(scope="module")
def ctx():
    from paper_2608_02611_b200 import binding
    c = binding.Context(0)
    yield c
    assert c.poll() == 0
    c.close()


def _call(ctx, k_cache, v_cache, slots=None):
    x = torch.arange(4 * HEADS * DIM, device=DEV).view(4, HEADS, DIM).remainder(97).bfloat16()
    slots = torch.tensor([0, 17, 33, 47], device=DEV) if slots is None else slots
    ctx.qk_norm_rope(x, x, norm=False, want_q=False, want_k=False, v=x + 1, k_cache=k_cache, v_cache=v_cache, slots=slots)
    return x, slots


@pytest.mark.parametrize("strides", [(2048, 0, 64, 1), (2048, 64, 64, 1), (0, 128, 64, 1), (64, 128, 64, 1), (2047, 128, 64, 1), (2048, 128, 63, 1),
                                     (2048, 127, 64, 1), (128, 128, 64, 1)])
def test_slots_that_overlap_are_refused(ctx, strides):
    from paper_2608_02611_b200.binding import KbError
    held = torch.zeros(PAGES * PAGE * HEADS * DIM, dtype=torch.bfloat16, device=DEV)
    bad = held.as_strided((PAGES, PAGE, HEADS, DIM), strides)
    good = torch.zeros(PAGES, PAGE, HEADS, DIM, dtype=torch.bfloat16, device=DEV)
    for pair in ((bad, good), (good, bad)):
        with pytest.raises(KbError):
            _call(ctx, *pair)
    assert not bool(held.any()) and not bool(good.any())


@pytest.mark.parametrize("order", [(0, 1, 2), (0, 2, 1), (1, 0, 2), (1, 2, 0), (2, 0, 1), (2, 1, 0)])
@pytest.mark.parametrize("gap", [0, 8])
def test_any_order_of_the_axes_is_taken(ctx, order, gap):
    """Pages, slots and heads in any order in memory, with gaps or without, keys and values side by side."""
    sizes = [(PAGES, PAGE, HEADS)[i] for i in order]
    held = torch.zeros(*sizes, 2, DIM + gap, dtype=torch.bfloat16, device=DEV)
    back = [order.index(i) for i in range(3)]
    k, v = (held[..., i, :DIM].permute(*back, 3) for i in (0, 1))
    x, slots = _call(ctx, k, v)
    assert torch.equal(k[slots // PAGE, slots % PAGE], x) and torch.equal(v[slots // PAGE, slots % PAGE], x + 1)
    assert int(held.ne(0).sum()) == int(x.ne(0).sum()) + int((x + 1).ne(0).sum())


def test_strides_of_axes_of_one_element_are_free(ctx):
    held = torch.zeros(2 * DIM, dtype=torch.bfloat16, device=DEV)
    x = torch.ones(1, 1, DIM, dtype=torch.bfloat16, device=DEV)
    k, v = (held[i * DIM:].as_strided((1, 1, 1, DIM), (0, 0, 0, 1)) for i in (0, 1))
    ctx.qk_norm_rope(x, x, norm=False, want_q=False, want_k=False, v=2 * x, k_cache=k, v_cache=v, slots=torch.zeros(1, dtype=torch.int64, device=DEV))
    assert bool((held[:DIM] == 1).all()) and bool((held[DIM:] == 2).all())
