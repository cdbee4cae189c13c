"""The rotation at far positions, against exact angles: within a few roundings of binary32 up to positions of 2^36, and within the
header's bound behind that."""
import math
from fractions import Fraction

import pytest
import torch

from tests import attention_exact as exact

pytestmark = pytest.mark.gpu
DEV = "cuda"
TWO_PI = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798214808651")
POSITIONS = [0, 1, -1, 10 ** 6, 2 ** 28 + 1, 2 ** 31 + 7, -2 ** 33 - 1, 2 ** 36 - 5, -2 ** 36, 2 ** 40 + 12345, 2 ** 50 - 3, -2 ** 57 + 1, 2 ** 63 - 1, -2 ** 63]


@pytest.mark.parametrize("dim", [16, 20])              # by vectors, and element by element
@pytest.mark.parametrize("interleaved", [False, True])
def test_angles_of_any_position(dim, interleaved):
    from paper_2608_02611_b200 import binding
    ctx = binding.Context(0)
    n = dim // 2
    f = torch.tensor([1.0, 0.3, 1e-4, 7.5, -2.25, 2.0 ** -30, 100.125, 3.14159, -1e-20, 2.0 ** 15][:n], dtype=torch.float64)
    pos = torch.tensor(POSITIONS)
    gen = torch.Generator()
    gen.manual_seed(5)
    x = torch.randn(len(POSITIONS), 3, dim, generator=gen).to(DEV)
    got, _ = ctx.qk_norm_rope(x, x, pos.to(DEV), f.to(DEV), norm=False, interleaved=interleaved)
    got, d = got.double().cpu(), x.double().cpu()
    a, b = (slice(0, None, 2), slice(1, None, 2)) if interleaved else (slice(0, n), slice(n, None))
    turns = [[(p * Fraction(float(w)) / TWO_PI) % 1 for w in f] for p in POSITIONS]
    angle = torch.tensor([[float(t * TWO_PI) for t in row] for row in turns], dtype=torch.float64)[:, None]
    want_a, want_b = (d[..., a] * angle.cos() - d[..., b] * angle.sin(), d[..., b] * angle.cos() + d[..., a] * angle.sin())
    # the header's bound on the angle, in radians; cosine and sine 4 u, two products and a sum 3 u, the angle's own rounding 1 u
    far = torch.tensor([[2 * math.pi * abs(p) * (2.0 ** -63 + 2.0 ** -74 * abs(float(w))) for w in f] for p in POSITIONS], dtype=torch.float64)[:, None]
    tol = (d[..., a].abs() + d[..., b].abs()) * (8 * exact.U + far)
    for want, at in ((want_a, a), (want_b, b)):
        err = (got[..., at] - want).abs()
        assert bool((err <= tol).all()), float((err / tol).max())
    assert ctx.poll() == 0
    ctx.close()
