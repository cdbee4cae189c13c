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


def test_a_norm_over_no_row_refuses_what_a_norm_over_rows_refuses(ctx):
    from paper_2608_02611_b200 import binding
    z = torch.empty(0, 256, device=DEV)
    w = torch.ones(256, device=DEV)
    for call in (lambda: ctx.layernorm(z, w, eps=0.0), lambda: ctx.layernorm(z, w, eps=float("inf")),
                 lambda: ctx.layernorm(z, w, quantize=torch.bfloat16), lambda: ctx.layernorm(z.int(), None),
                 lambda: ctx.layernorm(z, w, want_y=False, want_stats=False), lambda: ctx.layernorm(z[:, :0], None)):
        with pytest.raises(binding.KbError):
            call()
    r = ctx.layernorm(z, w, w, quantize=torch.float8_e5m2)
    assert r.y.shape == (0, 256) and r.mean.shape == (0,) and r.rstd.shape == (0,)
    assert r.q.shape == (0, 256) and r.q.dtype == torch.float8_e5m2 and r.scale.shape == (2, 0)
    only = ctx.layernorm(z.view(3, 0, 256), w, want_y=False)
    assert only.y is None and only.mean.shape == (0,)


def test_outputs_carry_no_gradient(ctx):
    """As documented: the operators take no part in autograd, whatever their inputs require."""
    x = torch.randn(8, 256, device=DEV, requires_grad=True)
    w = torch.ones(256, device=DEV, requires_grad=True)
    r = ctx.layernorm(x, w, quantize=torch.float8_e4m3fn)
    q, s = ctx.quantize_blocks(x)
    outs = [*r, q, s, ctx.matmul_blocks(q, s, q, s), *ctx.layernorm_backward(x, x, w, r.mean, r.rstd)]
    assert not any(o.requires_grad for o in outs)
    for call in (ctx.layernorm, ctx.layernorm_backward):
        assert "gradient" in call.__doc__
