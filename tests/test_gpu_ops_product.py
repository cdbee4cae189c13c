"""The 8-bit product at sizes that reach the kernel of CTA pairs (more tiles of 128 x 128 than the GPU has
SMs) and at contractions so long that every ring of the kernel for few rows goes round.

Each case asserts which kernel took it.  References and bounds are those of test_gpu_ops.py: 64 bits, and
the rounding errors of the contract.
"""
import pytest
import torch

from tests.test_gpu_ops import DEV, FLOATS, _operand, _product64, _product_bound, _scales, _within

pytestmark = pytest.mark.gpu

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2


@pytest.fixture(scope="module")
def ctx():
    from paper_2608_02611_b200 import binding
    c = binding.Context(0)
    yield c
    assert c.poll() == 0
    c.close()


def _case(M, N, K, tiles, ta=E4M3, tb=E4M3):
    kb = -(-K // 128)
    a, b = _operand(M, K, ta, 1), _operand(N, K, tb, 2)
    return a, _scales(kb, M, 3), b, _scales(kb, -(-N // 128) if tiles else N, 4)


# tiles of 256 x 256: 100 (two walks for some pairs, ten rows of tiles: more than the eight that
# neighbours share), 110, 66 on 33 columns, 80 on 40 rows; K blocks odd and even in number, whole and ragged
PAIR_SIZES = [(2500, 2401, 300), (2600, 2500, 1500), (300, 8200, 260), (10200, 511, 129), (2048, 2560, 256),
              (2305, 2050, 100), (2049, 2304, 1), (4097, 4100, 640), (130, 9500, 2700)]


@pytest.mark.parametrize("M,N,K", PAIR_SIZES)
@pytest.mark.parametrize("tiles", [True, False])
def test_product_by_pairs_against_64_bits(ctx, M, N, K, tiles):
    a, sa, b, sb = _case(M, N, K, tiles)
    want, size = _product64(a, sa, b, sb, tiles)
    for out in FLOATS:
        d = ctx.matmul_blocks(a, sa, b, sb, out_dtype=out)
        assert ctx.last_product == (256, 1)
        assert d.dtype == out
        _within(d, want, _product_bound(want, size, K, out))


@pytest.mark.parametrize("ta", [E4M3, E5M2])
@pytest.mark.parametrize("tb", [E4M3, E5M2])
@pytest.mark.parametrize("tiles", [True, False])
def test_product_by_pairs_of_either_format(ctx, ta, tb, tiles):
    M, N, K = 2050, 2305, 700
    a, sa, b, sb = _case(M, N, K, tiles, ta, tb)
    want, size = _product64(a, sa, b, sb, tiles)
    d = ctx.matmul_blocks(a, sa, b, sb, out_dtype=torch.float32)
    assert ctx.last_product == (256, 1)
    _within(d, want, _product_bound(want, size, K, torch.float32))


@pytest.mark.parametrize("M,N,K", [(2305, 2111, 300), (300, 8193, 150)])
@pytest.mark.parametrize("tiles", [True, False])
def test_product_by_pairs_writes_only_its_matrix(ctx, M, N, K, tiles):
    a, sa, b, sb = _case(M, N, K, tiles)
    want, size = _product64(a, sa, b, sb, tiles)
    for out in FLOATS:
        for gap in (1, 8, 24, -N % 8):
            held = torch.full((M + 2, N + gap), -3.0, dtype=out, device=DEV)
            got = ctx.matmul_blocks(a, sa, b, sb, out=held[1:-1, :N])
            assert ctx.last_product == (256, 1)
            _within(got, want, _product_bound(want, size, K, out))
            assert bool((held[0] == -3.0).all()) and bool((held[-1] == -3.0).all()) and bool((held[:, N:] == -3.0).all())


@pytest.mark.parametrize("tiles", [True, False])
def test_product_by_pairs_keeps_nonfinite_codes_to_their_rows_and_columns(ctx, tiles):
    M, N, K = 2305, 2111, 500
    a, sa, b, sb = _case(M, N, K, tiles, E4M3, E5M2)
    clean = ctx.matmul_blocks(a, sa, b, sb, out_dtype=torch.float32)
    a.view(torch.uint8)[M - 2, 17] = 0x7F            # NaN
    b.view(torch.uint8)[N - 3, K - 1] = 0x7C         # +Inf
    d = ctx.matmul_blocks(a, sa, b, sb, out_dtype=torch.float32)
    assert ctx.last_product == (256, 1)
    assert bool(d[M - 2].isnan().all()) and bool((~d[:, N - 3].isfinite()).all())
    d[M - 2], d[:, N - 3] = clean[M - 2], clean[:, N - 3]
    assert bool((d == clean).all())


def test_product_by_pairs_is_the_same_every_time(ctx):
    for tiles in (True, False):
        a, sa, b, sb = _case(2600, 2500, 1500, tiles)
        d = ctx.matmul_blocks(a, sa, b, sb, out_dtype=torch.float32)
        for _ in range(5):
            assert bool((ctx.matmul_blocks(a, sa, b, sb, out_dtype=torch.float32) == d).all())
        assert ctx.last_product == (256, 1)


# rows per tile, and K blocks per CTA past every ring's slots (nine, six or four stages, four accumulators,
# scales of sixteen blocks): by clusters of eight, by smaller ones, and by one CTA per tile
@pytest.mark.parametrize("M,N,K,rows,splits", [(1, 300, 20001, 16, 8), (20, 300, 32768, 32, 8), (50, 200, 24000, 64, 8),
                                               (100, 300, 20001, 128, 8), (1, 6000, 9000, 16, None),
                                               (60, 19200, 2600, 64, 1), (20, 18817, 2500, 32, 1), (100, 18817, 2700, 128, 1)])
@pytest.mark.parametrize("tiles", [True, False])
def test_product_of_few_rows_over_long_contractions(ctx, M, N, K, rows, splits, tiles):
    a, sa, b, sb = _case(M, N, K, tiles)
    want, size = _product64(a, sa, b, sb, tiles)
    for out in (torch.float32, torch.bfloat16):
        d = ctx.matmul_blocks(a, sa, b, sb, out_dtype=out)
        took, shared = ctx.last_product
        assert took == rows and (splits is None or shared == splits)
        assert -(-K // 128) // shared > 16
        _within(d, want, _product_bound(want, size, K, out))
        assert bool((ctx.matmul_blocks(a, sa, b, sb, out_dtype=out) == d).all())


SCALES = [2.0 ** e for e in (65, -72, -100, 112, -109, 127, -126, 90)]


@pytest.mark.parametrize("M,N,K,rows", [(5, 700, 500, 16), (20, 1100, 700, 32), (60, 900, 300, 64), (110, 1300, 500, 128),
                                        (2305, 2111, 500, 256), (2500, 2401, 1300, 256)])
@pytest.mark.parametrize("tiles", [True, False])
def test_product_with_scales_at_the_ends_of_the_range(ctx, M, N, K, rows, tiles):
    """Scales whose product, or whose product with a block's sum, leaves binary32 although the result does
    not: against 64 bits wherever the sum of magnitudes stays under 2^127.  Beside the usual bound, each of the
    kb additions and the products before it may lose 2^-150 to the smallest numbers."""
    a, sa, b, sb = _case(M, N, K, tiles)
    clean = ctx.matmul_blocks(a, sa, b, sb, out_dtype=torch.float32)
    step = 128 if tiles else 1
    touched_m, touched_n = torch.zeros(M, dtype=torch.bool, device=DEV), torch.zeros(N, dtype=torch.bool, device=DEV)
    sa, sb = sa.clone(), sb.clone()
    picks = sorted({min(M - 1, 1 + 37 * i) for i in range(2 * len(SCALES))})
    for i, m in enumerate(picks):
        sa[:, m] = SCALES[i % len(SCALES)]
        if M > 100:
            sa[i % sa.shape[0], m] = 0.01                  # one block of the row stays ordinary
        touched_m[m] = True
    a.view(torch.uint8)[picks[0]] = 0x80                   # codes of -0: sums of 0 under every scale
    a.view(torch.uint8)[picks[-1]] = 0x7E                  # the largest codes
    for i in range(len(SCALES)):
        n = min(sb.shape[1] - 1, i if tiles else 1 + 53 * i)
        sb[:, n] = SCALES[(3 * i + 1) % len(SCALES)]
        touched_n[n * step:(n + 1) * step] = True
    want, size = _product64(a, sa, b, sb, tiles)
    kb = -(-K // 128)
    for out in (torch.float32, torch.bfloat16):
        d = ctx.matmul_blocks(a, sa, b, sb, out_dtype=out)
        assert ctx.last_product[0] == rows
        inside = size < 2.0 ** 127
        assert bool(d[inside].isfinite().all())
        bound = _product_bound(want, size, K, out) + (kb + 2) * 2.0 ** -149
        _within(d[inside], want[inside], bound[inside])
        assert bool((d[picks[0]] == 0.0).all())
        if out == torch.float32:
            same = ~touched_m[:, None] & ~touched_n[None, :]
            assert bool((d[same] == clean[same]).all())
        assert bool((ctx.matmul_blocks(a, sa, b, sb, out_dtype=out)[inside] == d[inside]).all())


@pytest.mark.parametrize("ta", [E4M3, E5M2])
@pytest.mark.parametrize("tb", [E4M3, E5M2])
@pytest.mark.parametrize("M,N,K", [(2305, 2111, 500), (2200, 2400, 261)])
@pytest.mark.parametrize("scale,code", [((2.0 ** -70, 2.0 ** -71), 64.0), ((2.0 ** 99, 2.0 ** 29), 2.0 ** -6)])
def test_product_by_pairs_with_every_row_at_the_end_of_the_range(ctx, M, N, K, ta, tb, scale, code):
    """Tile scales whose product underflows or overflows for every row and block, with codes that bring the
    result back into the range: in every format, ragged in every direction, into rows at any alignment."""
    kb = -(-K // 128)
    a, b = _operand(M, K, ta, 1, code), _operand(N, K, tb, 2, code)
    sa = torch.full((kb, M), scale[0], device=DEV)
    sb = torch.full((kb, -(-N // 128)), scale[1], device=DEV)
    want, size = _product64(a, sa, b, sb, True)
    inside = size < 2.0 ** 127                             # elsewhere partial sums may overflow
    assert float(inside.double().mean()) > 0.1
    held = torch.full((M + 2, N + 3), -3.0, device=DEV)
    d = ctx.matmul_blocks(a, sa, b, sb, out=held[1:-1, :N])
    assert ctx.last_product == (256, 1)
    bound = _product_bound(want, size, K, torch.float32) + (kb + 2) * 2.0 ** -149
    _within(d[inside], want[inside], bound[inside])
    assert bool((held[0] == -3.0).all()) and bool((held[-1] == -3.0).all()) and bool((held[:, N:] == -3.0).all())
