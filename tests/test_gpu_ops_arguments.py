"""Arguments of the operators' Python calls that are refused before anything is launched."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx():
    from paper_2608_02611_b200 import binding
    c = binding.Context(0)
    yield c
    assert c.poll() == 0
    c.close()


class NoTruth:
    def __bool__(self):
        raise ValueError("neither true nor false")


def test_an_argument_without_a_truth_value_raises_its_own_error(ctx):
    x = torch.randn(8, 256, device=DEV)
    m, r = torch.zeros(8, device=DEV), torch.ones(8, device=DEV)
    before = ctx.launch_count
    for call in (lambda: ctx.quantize_blocks(x, tiles=NoTruth()), lambda: ctx.quantize_blocks(x, transpose=NoTruth()),
                 lambda: ctx.layernorm(x, want_y=NoTruth()), lambda: ctx.layernorm(x, want_stats=NoTruth()),
                 lambda: ctx.layernorm_backward(x, x, None, m, r, want_bias=NoTruth())):
        with pytest.raises(ValueError, match="neither"):
            call()
    assert ctx.launch_count == before
    with pytest.raises(TypeError):
        ctx.layernorm(x, eps="small")
