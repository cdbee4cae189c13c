"""Rows over very many keys."""
import math

import pytest
import torch

from tests.attention_exact import U

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx():
    from paper_2608_02611_b200 import binding
    c = binding.Context(0)
    yield c
    assert c.poll() == 0
    c.close()


@pytest.mark.parametrize("keys", [1 << 16, (1 << 17) + 5, 1 << 20])
@pytest.mark.parametrize("below", [0.25, 0.2, 0.1])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_a_long_rows_sum_takes_in_every_key(ctx, keys, below, dtype):
    """One key with the largest score, which the exponentials are relative to, and very many alike a little below it: where
    they are added one by one to the row's sum, each is rounded to the sum's steps in the same direction."""
    q, k = torch.zeros(130, 2, 8, dtype=dtype), torch.zeros(keys, 1, 8, dtype=dtype)
    q[..., 0] = 1.0
    k[1:, 0, 0] = -below
    s = float(k[1, 0, 0])
    want = math.log1p((keys - 1) * math.exp(s))
    k = k.to(DEV)
    lse = ctx.attention(q.to(DEV), k, k, torch.tensor([0, 130], dtype=torch.int32, device=DEV), torch.tensor([0, keys], dtype=torch.int32, device=DEV),
                        causal=False, scale=1.0, want_lse=True).lse.double().cpu()
    # additions: 32 in each half of a step, the steps, the halves; the exponent's rounding (below 16, so 16 u of it) and the exponential's 4 u;
    # the logarithm and its scaling 8 u of it
    bound = (32 + keys / 64 + 1 + 1 + 16 + 4) * U + 8 * U * want
    assert float((lse - want).abs().max()) <= bound


def test_the_most_keys_of_a_sequence_and_one_more(ctx):
    """2^24 keys: all of them count, and no wait runs out.  One more: refused, by the host without offsets, else by the device."""
    from paper_2608_02611_b200.binding import KbError
    most = 1 << 24
    k = torch.zeros(most + 1, 1, 8, dtype=torch.bfloat16, device=DEV)
    v = torch.ones_like(k)
    q = torch.ones(3, 1, 8, dtype=torch.bfloat16, device=DEV)
    r = ctx.attention(q, k[:most], v[:most], causal=False, want_lse=True)
    # equal scores: 128 for each key, and every sum is a power of two
    assert ctx.poll() == 0 and bool((r.out == 1.0).all())
    assert float((r.lse.double() - math.log(most)).abs().max()) <= 8 * U * math.log(most)
    with pytest.raises(KbError):
        ctx.attention(q, k, v, causal=False)
    out = torch.full_like(q, 5.0)
    offsets = [torch.tensor(o, dtype=torch.int32, device=DEV) for o in ([0, 2, 3], [0, most + 1, most + 1])]
    ctx.attention(q, k, v, *offsets, causal=False, out=out)
    assert ctx.poll() == 1 and ctx.poll() == 0
    assert bool((out[:2] == 5.0).all()) and bool((out[2] == 0.0).all())


def test_more_sequences_than_the_call_takes(ctx):
    from paper_2608_02611_b200.binding import KbError
    q = torch.ones(3, 1, 8, dtype=torch.bfloat16, device=DEV)
    offsets = torch.zeros((1 << 24) + 2, dtype=torch.int32, device=DEV)
    with pytest.raises(KbError):
        ctx.attention(q, q, q, offsets)
    offsets[-2:] = 3                                       # the last but one of 2^24 has the three tokens
    r = ctx.attention(q, q, q, offsets[1:], want_lse=True)
    assert ctx.poll() == 0 and torch.equal(r.out, ctx.attention(q, q, q).out)
