"""Layer norm, block quantisation and the 8-bit product against plain implementations in 64 bits.

Tolerances are bounds on the rounding errors of the definitions in include/kb_ops.h, u = 2^-24:
a sum of binary32 terms made of chains of at most k additions is off by at most k u sum|terms|;
storing a result rounds it once more to its type.  Quantisation is defined operation by operation
in binary32 and is compared bit for bit.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_ULP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}   # 24, 11 and 8 significant bits
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
FP8_MAX = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}
FLOATS = [torch.float32, torch.float16, torch.bfloat16]
DEV = "cuda"


@pytest.fixture(scope="module")
def ctx():
    from paper_2608_02611_b200 import binding
    c = binding.Context(0)
    yield c
    assert c.poll() == 0
    buffers, bad = c.check_guards()
    assert bad == 0
    c.close()


def _gen(seed):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    return g


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen)


def _strided(t, gap, offset=0):
    """The same matrix on the GPU with `gap` columns of NaN between rows, starting `offset`
    elements after an aligned address."""
    rows, cols = t.shape
    held = torch.full((rows * (cols + gap) + offset + 64,), float("nan"), device=DEV).to(t.dtype)
    view = held[offset:offset + rows * (cols + gap)].view(rows, cols + gap)[:, :cols]
    view.copy_(t)
    return view


def _within(got, want, bound):
    got, want = got.double().cpu(), want.double().cpu()
    err = (got - want).abs()
    ok = err <= bound.cpu()
    assert bool(ok.all()), f"{int((~ok).sum())} of {ok.numel()} beyond the bound, worst {float((err / bound.cpu()).max()):.3g} of it"


# ---- quantisation ---------------------------------------------------------------------------

def _blocks32(v, fp8, tiles):
    """The definition in binary32 on the CPU, with loops over blocks and nothing clever."""
    top = torch.tensor(FP8_MAX[fp8], dtype=torch.float32)
    v = v.float().cpu()
    R, C = v.shape
    kb = -(-C // 128)
    step = 128 if tiles else 1
    scale = torch.empty(kb, -(-R // step))
    code = torch.empty(R, C, dtype=torch.uint8)
    for b in range(kb):
        cols = slice(b * 128, min(C, b * 128 + 128))
        for r in range(0, R, step):
            blk = v[r:r + step, cols]
            fin = blk[blk.isfinite()].abs()
            a = torch.maximum(torch.tensor(2.0 ** -100), fin.max() if fin.numel() else torch.tensor(0.0))
            scale[b, r // step] = a / top
            t = (blk * 0.875) / (a * (0.875 / FP8_MAX[fp8]))      # the last factor is a power of two
            t = torch.minimum(torch.maximum(t, -top), top)
            t = torch.where(blk.isfinite(), t, torch.tensor(float("nan")))
            code[r:r + step, cols] = t.to(fp8).view(torch.uint8)
    return code, scale


def _same_codes(q, want, fp8):
    got = q.view(torch.uint8).cpu() if q.is_contiguous() else q.contiguous().view(torch.uint8).cpu()
    nan = want.view(fp8).float().isnan()
    assert bool((got.view(fp8).float().isnan() == nan).all())
    assert bool((got[~nan] == want[~nan]).all())


def _quant_input(rows, cols, dtype, seed):
    gen = _gen(seed)
    x = _randn(gen, rows, cols) * torch.exp(2.0 * _randn(gen, rows, 1))
    x[torch.rand(rows, cols, generator=gen) < 0.05] = 0.0
    return x.to(dtype)


QUANT_SIZES = [(1, 1), (1, 128), (3, 127), (8, 256), (5, 129), (130, 264), (128, 128), (257, 1000), (1, 5000), (600, 8)]


@pytest.mark.parametrize("rows,cols", QUANT_SIZES)
@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("fp8", [torch.float8_e4m3fn, torch.float8_e5m2])
def test_quantisation_bit_for_bit(ctx, rows, cols, tiles, transpose, fp8):
    for k, dtype in enumerate(FLOATS):
        x = _quant_input(rows, cols, dtype, rows * 1000 + cols + k)
        q, scale = ctx.quantize_blocks(x.to(DEV), fp8, tiles=tiles, transpose=transpose)
        code, want = _blocks32(x.t() if transpose else x, fp8, tiles)
        assert scale.shape == want.shape and bool((scale.cpu() == want).all())
        _same_codes(q, code, fp8)


@pytest.mark.parametrize("tiles,transpose", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("fp8", [torch.float8_e4m3fn, torch.float8_e5m2])
def test_quotients_halfway_between_two_codes_go_to_the_even_one(ctx, tiles, transpose, fp8):
    """16-bit inputs make quotients V F / a that lie exactly between two codes: against the definition
    in 64 bits, code for code, with largest values of every bf16 significand."""
    top = FP8_MAX[fp8]
    sig = torch.arange(128, 256, dtype=torch.float64)
    x = torch.zeros(128, 128, dtype=torch.float64)
    x[:, :] = sig[None, :] * torch.exp2(-torch.arange(128)[:, None] % 9).double()
    for amax in range(128, 256, 3):
        v = torch.minimum(x, torch.tensor(float(amax)).double())
        v[:, 0] = v[0, :] = amax
        q, _ = ctx.quantize_blocks(v.to(torch.bfloat16).to(DEV), fp8, tiles=tiles, transpose=transpose)
        t = (v.t() if transpose else v) * top / amax
        bits, low = (3, -6) if fp8 == torch.float8_e4m3fn else (2, -14)
        step = torch.exp2(torch.floor(torch.log2(t)).clamp_min(low) - bits)
        want = torch.round(t / step) * step
        assert bool((q.double().cpu() == want).all())


@pytest.mark.parametrize("tiles,transpose", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("fp8", [torch.float8_e4m3fn, torch.float8_e5m2])
def test_quotients_of_the_smallest_and_largest_blocks(ctx, tiles, transpose, fp8):
    """The same with largest values of 2^-100 to 2^-90, around 2^-60 and at the top of the range, and quotients
    down to half the smallest code: neither the division nor its remainder may lose bits to binary32's range."""
    top = FP8_MAX[fp8]
    bits, low, steps = (3, -6, 20) if fp8 == torch.float8_e4m3fn else (2, -14, 34)
    sig = torch.arange(128, 256, dtype=torch.float64)
    for e in [*range(-100, -89), -70, -61, -60, 100, 126, 127]:
        x = sig[None, :] * torch.exp2(float(e - 7) - (torch.arange(128)[:, None] % steps).double())
        for m in (*range(128, 256, 9), 167, 224, 231):
            amax = m * 2.0 ** (e - 7)
            v = torch.minimum(x, torch.tensor(amax).double())
            v[:, 0] = v[0, :] = amax
            v = v.to(torch.bfloat16)                        # the smallest lose bits to the type, before the call
            q, scale = ctx.quantize_blocks(v.to(DEV), fp8, tiles=tiles, transpose=transpose)
            assert bool((scale.cpu() == (torch.tensor(amax, dtype=torch.float32) / top)).all())
            t = (v.t() if transpose else v).double() * top / amax
            step = torch.exp2(torch.floor(torch.log2(t.clamp_min(2.0 ** -60))).clamp_min(low) - bits)
            assert bool((q.double().cpu() == torch.round(t / step) * step).all()), (e, m)


@pytest.mark.parametrize("exponent", [-100, -97, -80, -62, -59])
@pytest.mark.parametrize("fp8", [torch.float8_e4m3fn, torch.float8_e5m2])
def test_quantisation_of_tiny_binary32_blocks_bit_for_bit(ctx, exponent, fp8):
    """Elements down to and below binary32's smallest normal value, in blocks of tiny largest values."""
    gen = _gen(exponent + 200)
    x = torch.rand(64, 256, generator=gen) * torch.exp2(-40.0 * torch.rand(64, 256, generator=gen)) * 2.0 ** exponent
    x[:, ::2].neg_()
    x[:, ::128] = 1.3 * 2.0 ** exponent
    q, scale = ctx.quantize_blocks(x.to(DEV), fp8)
    want = _blocks32(x, fp8, False)[1]
    code = _blocks32(x * 2.0 ** 40 if exponent < -60 else x, fp8, False)[0]
    assert bool((scale.cpu() == want).all())
    _same_codes(q, code, fp8)


@pytest.mark.parametrize("gap,offset", [(8, 0), (3, 0), (0, 1), (5, 3)])
@pytest.mark.parametrize("tiles,transpose", [(False, False), (False, True), (True, False), (True, True)])
def test_quantisation_of_strided_and_unaligned_rows(ctx, gap, offset, tiles, transpose):
    for dtype in FLOATS:
        x = _quant_input(70, 392, dtype, 5)
        q, scale = ctx.quantize_blocks(_strided(x, gap, offset), tiles=tiles, transpose=transpose)
        code, want = _blocks32(x.t() if transpose else x, torch.float8_e4m3fn, tiles)
        assert bool((scale.cpu() == want).all())
        _same_codes(q, code, torch.float8_e4m3fn)


@pytest.mark.parametrize("rows,cols", [(1, 5), (3, 131), (37, 1001), (129, 515)])
@pytest.mark.parametrize("gap,offset", [(0, 0), (0, 1), (0, 3), (1, 5), (6, 7)])
@pytest.mark.parametrize("tiles,transpose", [(False, False), (True, False), (False, True)])
def test_quantisation_of_rows_at_every_alignment(ctx, rows, cols, gap, offset, tiles, transpose):
    """The granules of 16 bytes that a row shares with its neighbours, and with what lies before and
    behind the matrix, hold NaN."""
    for dtype in FLOATS:
        x = _quant_input(rows, cols, dtype, rows + cols)
        q, scale = ctx.quantize_blocks(_strided(x, gap, offset), tiles=tiles, transpose=transpose)
        code, want = _blocks32(x.t() if transpose else x, torch.float8_e4m3fn, tiles)
        assert bool((scale.cpu() == want).all())
        _same_codes(q, code, torch.float8_e4m3fn)


@pytest.mark.parametrize("cols", [384, 300])
@pytest.mark.parametrize("tiles,transpose", [(False, False), (False, True), (True, False), (True, True)])
def test_quantisation_of_nonfinite_zero_and_extreme_blocks(ctx, cols, tiles, transpose):
    """NaN and Inf become NaN and leave the block's scale alone; empty (all-zero or all-NaN) blocks
    and blocks at both ends of the binary32 range keep finite scales."""
    x = _quant_input(256, cols, torch.float32, 11)
    x[:128, :128] = 0.0
    x[128:, :128] = float("nan")
    x[3, 130] = float("inf")
    x[200, 131] = float("-inf")
    x[7, 256:] = float("nan")
    x[9, 257] = 3.4e38
    x[130, 260] = 1e-42
    for fp8 in FP8_MAX:
        q, scale = ctx.quantize_blocks(x.to(DEV), fp8, tiles=tiles, transpose=transpose)
        code, want = _blocks32(x.t() if transpose else x, fp8, tiles)
        assert bool(scale.isfinite().all()) and bool((scale.cpu() == want).all())
        _same_codes(q, code, fp8)


def test_quantisation_writes_nothing_outside(ctx):
    from paper_2608_02611_b200 import binding
    L = binding.load()
    x = _quant_input(130, 200, torch.bfloat16, 3).to(DEV)
    for tiles in (0, 1):
        for transpose in (0, 1):
            R, C = (200, 130) if transpose else (130, 200)
            held = torch.full((R + 2, 208), 0xEE, dtype=torch.uint8, device=DEV)
            n = -(-C // 128) * (-(-R // 128) if tiles else R)
            scale = torch.full((n + 16,), -7.0, device=DEV)
            rc = L.kb_quantize_blocks(ctx._h, x.data_ptr(), 130, 200, 200, binding.KB_BF16, transpose, tiles,
                                      held[1:].data_ptr(), 208, binding.KB_F8E4M3, scale[8:].data_ptr(),
                                      torch.cuda.current_stream().cuda_stream)
            assert rc == 0
            torch.cuda.synchronize()
            assert bool((held[0] == 0xEE).all()) and bool((held[-1] == 0xEE).all()) and bool((held[:, C:] == 0xEE).all())
            assert bool((scale[:8] == -7.0).all()) and bool((scale[8 + n:] == -7.0).all())
            assert bool((scale[8:8 + n] > 0.0).all())


# ---- layer norm ---------------------------------------------------------------------------------

def _norm_input(rows, cols, dtype, seed):
    gen = _gen(seed)
    x = (_randn(gen, rows, cols) * torch.exp(0.5 * _randn(gen, cols)) + 2.0 * _randn(gen, rows, 1)).to(dtype)
    w, b = 1.0 + 0.2 * _randn(gen, cols), 0.2 * _randn(gen, cols)
    return x, w, b


def _norm64(x, w, b, eps):
    x = x.double()
    mean = x.mean(1)
    var = (x - mean[:, None]).square().mean(1)
    rstd = 1.0 / torch.sqrt(var + eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    return xh * w.double() + b.double(), mean, rstd, xh


def _chain(cols):
    """Longest chain of additions of a row's sum: a lane's elements, then the warps' trees."""
    return 64 + cols // 512


NORM_SIZES = [(1, 1), (2, 7), (1, 8192), (3, 256), (5, 257), (33, 1000), (7, 1024), (4, 1032), (9, 2049), (300, 4096),
              (2, 16384), (3, 16400), (2, 32768), (2, 40001), (1, 70000)]


@pytest.mark.parametrize("rows,cols", NORM_SIZES)
@pytest.mark.parametrize("dtype", FLOATS)
def test_layernorm_against_64_bits(ctx, rows, cols, dtype):
    for param in {dtype, torch.float32}:
        x, w, b = _norm_input(rows, cols, dtype, rows * 7 + cols)
        w, b = w.to(param), b.to(param)
        eps = 1e-5
        r = ctx.layernorm(x.to(DEV), w.to(DEV), b.to(DEV), eps)
        y, mean, rstd, xh = _norm64(x, w, b, eps)
        k = _chain(cols)
        size = x.double().abs().mean(1)
        _within(r.mean, mean, (k + 2) * U * size + TINY[torch.float32])
        # the variance: its own sum, and the mean's error squared over the variance (far smaller)
        mean_err = (k + 2) * U * size * rstd
        rstd_err = (k + 8) * U + mean_err.square()
        _within(r.rstd, rstd, rstd_err * rstd)
        bound = w.double().abs() * (mean_err[:, None] + xh.abs() * (rstd_err[:, None] + 4 * U)) + 2 * U * (y.abs() + b.double().abs())
        _within(r.y, y, bound * (1 + HALF_ULP[dtype]) + HALF_ULP[dtype] * y.abs() + TINY[dtype])


@pytest.mark.parametrize("rows,cols,dtype", [(5000, 1032, torch.bfloat16), (4001, 4096, torch.bfloat16),
                                             (3700, 2056, torch.float16), (1800, 8192, torch.float32),
                                             (1500, 16384, torch.bfloat16)])
def test_layernorm_and_backward_of_many_rows(ctx, rows, cols, dtype):
    """Rows enough for the walks that read ahead, in matrices whose rows lie apart."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(rows)
    held = torch.full((rows, cols + 8), float("nan"), device=DEV).to(dtype)
    x = held[:, :cols]
    x.copy_(torch.randn(rows, cols, generator=gen, device=DEV) + 2.0 * torch.randn(rows, 1, generator=gen, device=DEV))
    w, b = (1.0 + 0.2 * torch.randn(cols, generator=gen, device=DEV)).to(dtype), torch.randn(cols, generator=gen, device=DEV).to(dtype)
    r = ctx.layernorm(x, w, b, quantize=torch.float8_e4m3fn)
    y, mean, rstd, xh = _norm64(x, w, b, 1e-5)
    k = _chain(cols)
    mean_err = (k + 2) * U * x.double().abs().mean(1) * rstd
    rstd_err = (k + 8) * U + mean_err.square()
    _within(r.rstd, rstd, rstd_err * rstd)
    bound = w.double().abs() * (mean_err[:, None] + xh.abs() * (rstd_err[:, None] + 4 * U)) + 2 * U * (y.abs() + b.double().abs())
    _within(r.y, y, bound * (1 + HALF_ULP[dtype]) + HALF_ULP[dtype] * y.abs() + TINY[dtype])
    pad = -cols % 128
    amax = torch.nn.functional.pad(y, (0, pad)).abs().view(rows, -1, 128).amax(2).t()
    _within(r.scale, amax / 448.0, 2.0 ** -14 * amax / 448.0)
    s = r.scale.double().t().repeat_interleave(128, 1)[:, :cols]
    _within(r.q.double() * s, y, (2.0 ** -4 * y.abs() + 2.0 ** -10 * s) * 1.001 + 1e-4)
    dy = (0.1 * torch.randn(rows, cols, generator=gen, device=DEV)).to(dtype)
    dx, dw, db = ctx.layernorm_backward(dy, x, w, r.mean, r.rstd)
    want_dx, want_dw, want_db, xh, g = _bwd64(dy, x, w, r.mean, r.rstd)
    bound = r.rstd.double()[:, None] * ((k + 8) * U * (g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True)) + 8 * U * g.abs())
    _within(dx, want_dx, 1.01 * bound + HALF_ULP[dtype] * want_dx.abs() + TINY[dtype])
    rk = 128 + rows
    _within(dw, want_dw, 1.01 * rk * U * (dy.double() * xh).abs().sum(0) + HALF_ULP[dtype] * want_dw.abs() + TINY[dtype])
    _within(db, want_db, 1.01 * rk * U * dy.double().abs().sum(0) + HALF_ULP[dtype] * want_db.abs() + TINY[dtype])


@pytest.mark.parametrize("gap,offset", [(8, 0), (1, 0), (0, 1), (5, 3)])
def test_layernorm_of_strided_and_unaligned_rows(ctx, gap, offset):
    for dtype in FLOATS:
        for cols in (776, 3000):
            x, w, b = _norm_input(20, cols, dtype, cols)
            r = ctx.layernorm(_strided(x, gap, offset), w.to(dtype).to(DEV), b.to(dtype).to(DEV), quantize=torch.float8_e4m3fn)
            s = ctx.layernorm(x.to(DEV).contiguous(), w.to(dtype).to(DEV), b.to(dtype).to(DEV), quantize=torch.float8_e4m3fn)
            y, mean, rstd, xh = _norm64(x, w.to(dtype), b.to(dtype), 1e-5)
            # the order of the sums may differ with the layout, by no more than their bound
            k = _chain(cols)
            err = (k + 2) * U * x.double().abs().mean(1) * rstd
            bound = w.double().abs() * (err[:, None] + xh.abs() * ((k + 12) * U + err.square()[:, None])) + 2 * U * (y.abs() + 1)
            _within(r.y, y, 1.01 * bound + HALF_ULP[dtype] * y.abs() + TINY[dtype])
            assert r.q.shape == s.q.shape and r.scale.shape == s.scale.shape
            _within(r.scale, s.scale, 2.0 ** -16 * s.scale.double())


@pytest.mark.parametrize("rows,cols", [(1, 128), (3, 1000), (5, 1024), (130, 2048), (2, 5001), (2, 20000), (1, 40000)])
@pytest.mark.parametrize("fp8", [torch.float8_e4m3fn, torch.float8_e5m2])
def test_layernorm_hands_over_blocks(ctx, rows, cols, fp8):
    """The fused blocks are those of the binary32 y: with an fp32 row they are, bit for bit, what
    quantize_blocks makes of the y that the same call returns."""
    x, w, b = _norm_input(rows, cols, torch.float32, cols)
    r = ctx.layernorm(x.to(DEV), w.to(DEV), b.to(DEV), quantize=fp8)
    q, scale = ctx.quantize_blocks(r.y, fp8)
    assert bool((r.scale == scale).all())
    assert bool((r.q.contiguous().view(torch.uint8) == q.contiguous().view(torch.uint8)).all())
    only = ctx.layernorm(x.to(DEV), w.to(DEV), b.to(DEV), want_y=False, want_stats=False, quantize=fp8)
    assert only.y is None and only.mean is None
    assert bool((only.q.contiguous().view(torch.uint8) == q.contiguous().view(torch.uint8)).all())
    # for a 16-bit row: each code times its scale is within half a step of the unrounded y
    for dtype in (torch.float16, torch.bfloat16):
        xd = x.to(dtype)
        r = ctx.layernorm(xd.to(DEV), w.to(DEV), b.to(DEV), want_y=False, quantize=fp8)
        y = _norm64(xd, w, b, 1e-5)[0]
        s = r.scale.double().cpu().t().repeat_interleave(128, 1)[:, :cols]
        step = 2.0 ** (-4 if fp8 == torch.float8_e4m3fn else -3)
        low = 2.0 ** (-10 if fp8 == torch.float8_e4m3fn else -17)      # half of the smallest step
        _within(r.q.double().cpu() * s, y, step * y.abs() * 1.001 + low * s + 1e-4)


def test_layernorm_rows_are_independent_of_nonfinite_neighbours(ctx):
    x, w, b = _norm_input(6, 2000, torch.bfloat16, 1)
    clean = ctx.layernorm(x.to(DEV), w.to(DEV), b.to(DEV), quantize=torch.float8_e4m3fn)
    x[1, 5] = float("nan")
    x[3, 1999] = float("inf")
    r = ctx.layernorm(x.to(DEV), w.to(DEV), b.to(DEV), quantize=torch.float8_e4m3fn)
    for row in range(6):
        if row in (1, 3):
            assert bool(r.y[row].isnan().all()) and bool(r.q[row].float().isnan().all()) and bool(r.scale[:, row].isfinite().all())
        else:
            assert bool((r.y[row] == clean.y[row]).all()) and bool((r.scale[:, row] == clean.scale[:, row]).all())


def test_layernorm_of_constant_rows_and_without_parameters(ctx):
    x = torch.full((3, 777), 1234.5, device=DEV)
    r = ctx.layernorm(x)
    assert bool((r.y == 0.0).all()) and bool((r.mean == 1234.5).all())
    assert bool((r.rstd - 1e-5 ** -0.5).abs().max() < 1e-4 * 1e-5 ** -0.5)
    w = torch.randn(777, device=DEV)
    assert bool((ctx.layernorm(x, None, w).y == w).all())


def _bwd64(dy, x, w, mean, rstd):
    dy, x, w = dy.double(), x.double(), w.double()
    mean, rstd = mean.double()[:, None], rstd.double()[:, None]
    xh = (x - mean) * rstd
    g = dy * w
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0), xh, g


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 300), (3, 7), (40, 256), (700, 513), (65, 1000), (9, 1032), (310, 4096), (17, 4100),
                                       (5, 8192), (6, 8200), (40, 10001), (3, 20000)])
@pytest.mark.parametrize("dtype", FLOATS)
def test_layernorm_backward_against_64_bits(ctx, rows, cols, dtype):
    for param in {dtype, torch.float32}:
        x, w, b = _norm_input(rows, cols, dtype, rows + cols)
        w = w.to(param)
        dy = (0.1 * _randn(_gen(cols), rows, cols) + 0.01).to(dtype)
        _, mean, rstd, _ = _norm64(x, w, b, 1e-5)
        mean, rstd = mean.float(), rstd.float()
        dx, dw, db = ctx.layernorm_backward(dy.to(DEV), x.to(DEV), w.to(DEV), mean.to(DEV), rstd.to(DEV))
        assert dw.dtype == param and db.dtype == param and dx.dtype == dtype
        want_dx, want_dw, want_db, xh, g = _bwd64(dy, x, w, mean, rstd)
        k = _chain(cols)
        ga, gx = g.abs(), (g * xh).abs()
        bound = rstd.double()[:, None] * ((k + 8) * U * (ga.mean(1, keepdim=True) + xh.abs() * gx.mean(1, keepdim=True)) + 8 * U * ga)
        _within(dx, want_dx, 1.01 * bound + HALF_ULP[dtype] * want_dx.abs() + TINY[dtype])
        rk = 128 + rows
        _within(dw, want_dw, 1.01 * rk * U * (dy.double() * xh).abs().sum(0) + HALF_ULP[param] * want_dw.abs() + TINY[param])
        _within(db, want_db, 1.01 * rk * U * dy.double().abs().sum(0) + HALF_ULP[param] * want_db.abs() + TINY[param])


def test_layernorm_backward_against_differences(ctx):
    """Central differences of sum(dy * y) in 64 bits, in every direction of x, weight and bias."""
    rows, cols, eps, h = 3, 20, 1e-5, 1e-6
    x, w, b = _norm_input(rows, cols, torch.float32, 9)
    dy = _randn(_gen(2), rows, cols)
    r = ctx.layernorm(x.to(DEV), w.to(DEV), b.to(DEV), eps)
    dx, dw, db = ctx.layernorm_backward(dy.to(DEV), x.to(DEV), w.to(DEV), r.mean, r.rstd)

    def loss(x, w, b):
        return float((_norm64(x, w, b, eps)[0] * dy.double()).sum())

    def slope(k, i):
        args = [x.double().clone(), w.double().clone(), b.double().clone()]
        args[k].view(-1)[i] += h
        up = loss(*args)
        args[k].view(-1)[i] -= 2 * h
        return (up - loss(*args)) / (2 * h)

    for k, got in enumerate((dx, dw, db)):
        want = torch.tensor([slope(k, i) for i in range(got.numel())]).view(got.shape)
        # differences: h^2 and 1e-16/h, below 1e-8 here; binary32 gradients: a few hundred u of terms of order 1
        assert float((got.double().cpu() - want).abs().max()) < 512 * U * float(want.abs().max() + 1)


def test_layernorm_backward_strided_partial_outputs_and_repeats(ctx):
    from paper_2608_02611_b200 import binding
    for dtype in FLOATS:
        x, w, b = _norm_input(50, 1500, dtype, 4)
        dy = _randn(_gen(5), 50, 1500).to(dtype)
        r = ctx.layernorm(x.to(DEV), w.to(DEV), b.to(DEV))
        first = ctx.layernorm_backward(_strided(dy, 4), _strided(x, 12), w.to(DEV), r.mean, r.rstd)
        again = ctx.layernorm_backward(_strided(dy, 4), _strided(x, 12), w.to(DEV), r.mean, r.rstd)
        for p, q in zip(first, again):
            assert bool((p == q).all())
        none = ctx.layernorm_backward(_strided(dy, 4), _strided(x, 12), w.to(DEV), r.mean, r.rstd, want_bias=False)
        assert none[2] is None and bool((none[1] == first[1]).all())
        dw = torch.empty(1500, device=DEV)
        dyd, xd = dy.to(DEV), x.to(DEV)
        rc = binding.load().kb_layernorm_backward(
            ctx._h, dyd.data_ptr(), 1500, xd.data_ptr(), 1500, 50, 1500, binding.DTYPE_CODE[dtype], None,
            binding.KB_F32, r.mean.data_ptr(), r.rstd.data_ptr(), None, 0, dw.data_ptr(), None,
            torch.cuda.current_stream().cuda_stream)
        assert rc == 0
        _, want, _, xh, _ = _bwd64(dy, x, torch.ones(1500), r.mean.cpu(), r.rstd.cpu())
        _within(dw, want, (128 + 50 + 4) * U * (dy.double() * xh).abs().sum(0))


def test_layernorm_backward_broadcast_over_many_rows(ctx):
    """The parameters' gradients sum over every row: more rows than the grid has places."""
    rows, cols = 20000, 96
    x, w, b = _norm_input(rows, cols, torch.bfloat16, 6)
    dy = _randn(_gen(7), rows, cols).to(torch.bfloat16)
    _, mean, rstd, _ = _norm64(x, w, b, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    dx, dw, db = ctx.layernorm_backward(dy.to(DEV), x.to(DEV), w.to(DEV), mean.to(DEV), rstd.to(DEV))
    _, want_dw, want_db, xh, _ = _bwd64(dy, x, w, mean, rstd)
    _within(dw, want_dw, 256 * U * (dy.double() * xh).abs().sum(0))
    _within(db, want_db, 256 * U * dy.double().abs().sum(0))


# ---- product ---------------------------------------------------------------------------------------

def _operand(rows, cols, fp8, seed, scale=1.0):
    """Codes with every exponent in use, rows padded with NaN codes to a 16-byte stride + 16."""
    gen = _gen(seed)
    v = (_randn(gen, rows, cols) * torch.exp(1.5 * _randn(gen, rows, cols)) * scale).clamp(-400, 400)
    ld = (cols + 15) // 16 * 16 + 16
    held = torch.full((rows, ld), 0x7F, dtype=torch.uint8)
    held[:, :cols] = v.to(fp8).view(torch.uint8)
    return held.to(DEV).view(fp8)[:, :cols]


def _scales(kb, n, seed):
    return torch.exp(_randn(_gen(seed), kb, n)).to(DEV) * 0.01


def _product64(a, sa, b, sb, tiles):
    K = a.shape[1]
    k = torch.arange(K, device=DEV) // 128
    n = torch.arange(b.shape[0], device=DEV) // (128 if tiles else 1)
    a64, b64 = a.double() * sa.double()[k].t(), b.double() * sb.double()[k][:, n].t()
    return a64 @ b64.t(), a64.abs() @ b64.abs().t()


def _product_bound(want, size, K, out):
    # per block the tensor cores add 128 products, each addition off by 2^-23 of the sum of
    # magnitudes at most (truncation); then a product and an addition per block, and the rounding
    kb = -(-K // 128)
    return (128 * 2.0 ** -23 + (kb + 12) * U) * size * 1.01 + HALF_ULP[out] * want.abs() + TINY[out]


MM_SIZES = [(1, 1, 1), (1, 128, 128), (1, 1000, 1030), (2, 129, 127), (16, 256, 512), (17, 300, 4096), (33, 128, 129),
            (64, 640, 2000), (65, 130, 257), (128, 128, 128), (129, 257, 1000), (200, 513, 640), (256, 256, 256),
            (257, 1025, 400), (512, 512, 1024), (1000, 777, 333), (4096, 8, 512), (700, 2100, 260)]


@pytest.mark.parametrize("M,N,K", MM_SIZES)
@pytest.mark.parametrize("tiles", [True, False])
def test_product_against_64_bits(ctx, M, N, K, tiles):
    kb = -(-K // 128)
    a, b = _operand(M, K, torch.float8_e4m3fn, 1), _operand(N, K, torch.float8_e4m3fn, 2)
    sa, sb = _scales(kb, M, 3), _scales(kb, -(-N // 128) if tiles else N, 4)
    want, size = _product64(a, sa, b, sb, tiles)
    for out in FLOATS:
        d = ctx.matmul_blocks(a, sa, b, sb, out_dtype=out)
        assert d.dtype == out
        _within(d, want, _product_bound(want, size, K, out))


@pytest.mark.parametrize("ta", [torch.float8_e4m3fn, torch.float8_e5m2])
@pytest.mark.parametrize("tb", [torch.float8_e4m3fn, torch.float8_e5m2])
@pytest.mark.parametrize("M", [3, 100, 600])
def test_product_of_either_format(ctx, ta, tb, M):
    N, K = 300, 700
    a, b = _operand(M, K, ta, 1), _operand(N, K, tb, 2)
    sa, sb = _scales(6, M, 3), _scales(6, 3, 4)
    want, size = _product64(a, sa, b, sb, True)
    _within(ctx.matmul_blocks(a, sa, b, sb, out_dtype=torch.float32), want, _product_bound(want, size, K, torch.float32))


@pytest.mark.parametrize("M,N", [(5, 300), (70, 300), (600, 520)])
def test_product_keeps_nonfinite_codes_to_their_rows_and_columns(ctx, M, N):
    K = 500
    a, b = _operand(M, K, torch.float8_e4m3fn, 1), _operand(N, K, torch.float8_e5m2, 2)
    sa, sb = _scales(4, M, 3), _scales(4, N, 4)
    clean = ctx.matmul_blocks(a, sa, b, sb, out_dtype=torch.float32)
    a.view(torch.uint8)[M - 2, 17] = 0x7F            # NaN
    b.view(torch.uint8)[N - 3, K - 1] = 0x7C         # +Inf
    d = ctx.matmul_blocks(a, sa, b, sb, out_dtype=torch.float32)
    assert bool(d[M - 2].isnan().all())
    assert bool((~d[:, N - 3].isfinite()).all())
    rows = [i for i in range(M) if i != M - 2]
    cols = [j for j in range(N) if j != N - 3]
    assert bool((d[rows][:, cols] == clean[rows][:, cols]).all())


@pytest.mark.parametrize("M,N,K", [(1, 200, 300), (40, 130, 130), (300, 500, 200), (520, 770, 300)])
def test_product_writes_only_its_matrix(ctx, M, N, K):
    a, b = _operand(M, K, torch.float8_e4m3fn, 1), _operand(N, K, torch.float8_e4m3fn, 2)
    kb = -(-K // 128)
    sa, sb = _scales(kb, M, 3), _scales(kb, N, 4)
    want, size = _product64(a, sa, b, sb, False)
    for out in FLOATS:
        for gap in (1, 8, 24):
            held = torch.full((M + 2, N + gap), -3.0, dtype=out, device=DEV)
            got = ctx.matmul_blocks(a, sa, b, sb, out=held[1:-1, :N])
            _within(got, want, _product_bound(want, size, K, out))
            assert bool((held[0] == -3.0).all()) and bool((held[-1] == -3.0).all()) and bool((held[:, N:] == -3.0).all())


def test_product_is_the_same_every_time(ctx):
    for M, N, K in ((1, 512, 4096), (130, 1000, 2048), (600, 600, 1000)):
        a, b = _operand(M, K, torch.float8_e4m3fn, 1), _operand(N, K, torch.float8_e4m3fn, 2)
        kb = -(-K // 128)
        sa, sb = _scales(kb, M, 3), _scales(kb, -(-N // 128), 4)
        d = ctx.matmul_blocks(a, sa, b, sb, out_dtype=torch.float32)
        for _ in range(5):
            assert bool((ctx.matmul_blocks(a, sa, b, sb, out_dtype=torch.float32) == d).all())


def test_empty_operands(ctx):
    z = torch.empty((0, 256), dtype=torch.bfloat16, device=DEV)
    w = torch.ones(256, dtype=torch.bfloat16, device=DEV)
    assert ctx.layernorm(z, w, w).y.shape == (0, 256)
    dx, dw, db = ctx.layernorm_backward(z, z, w, torch.empty(0, device=DEV), torch.empty(0, device=DEV))
    assert dx.shape == (0, 256) and bool((dw == 0).all()) and bool((db == 0).all())
    q, s = ctx.quantize_blocks(z)
    assert q.shape == (0, 256) and s.shape == (2, 0)
    qt, st = ctx.quantize_blocks(z, transpose=True)
    assert qt.shape == (256, 0) and st.shape == (0, 256)
    b, sb = ctx.quantize_blocks(torch.ones(128, 256, dtype=torch.bfloat16, device=DEV), tiles=True)
    assert ctx.matmul_blocks(q, s, b, sb).shape == (0, 128)
    # no token: the weight's gradient is zero
    d = ctx.matmul_blocks(qt, st, qt, st, out_dtype=torch.float32)
    assert d.shape == (256, 256) and bool((d == 0).all())


def test_a_training_step_in_8_bits(ctx):
    """Norm, product and all three gradients chained through the public calls, on a stream of
    their own, against the same step in 64 bits on the dequantised operands."""
    T, C, N = 200, 384, 512
    x, w, b = _norm_input(T, C, torch.bfloat16, 1)
    x, w, b = x.to(DEV), w.to(DEV), b.to(DEV)
    W = (0.05 * _randn(_gen(3), N, C)).to(torch.bfloat16).to(DEV)
    dY = (0.1 * _randn(_gen(4), T, N)).to(torch.bfloat16).to(DEV)

    def undo(q, s, tiles=False):
        s = s.double().t()
        s = s.repeat_interleave(128, 0)[:q.shape[0]] if tiles else s
        return q.double() * s.repeat_interleave(128, 1)[:, :q.shape[1]]

    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        h = ctx.layernorm(x, w, b, quantize=torch.float8_e4m3fn)
        wq, ws = ctx.quantize_blocks(W, tiles=True)
        y = ctx.matmul_blocks(h.q, h.scale, wq, ws)
        wtq, wts = ctx.quantize_blocks(W, tiles=True, transpose=True)
        gq, gs = ctx.quantize_blocks(dY, torch.float8_e5m2)
        dh = ctx.matmul_blocks(gq, gs, wtq, wts)
        gtq, gts = ctx.quantize_blocks(dY, torch.float8_e5m2, transpose=True)
        htq, hts = ctx.quantize_blocks(h.y, transpose=True)
        dW = ctx.matmul_blocks(gtq, gts, htq, hts, out_dtype=torch.float32)
        dx, dw, db = ctx.layernorm_backward(dh, x, w, h.mean, h.rstd)
    stream.synchronize()
    assert bool((wts == ws.t()).all()) and bool((wtq.view(torch.uint8) == wq.view(torch.uint8).t()).all())

    def near(got, p, q, u):
        want, size = p @ q.t(), p.abs() @ q.abs().t()
        _within(got, want, 2.0 ** -15 * size + u * want.abs())

    near(y, undo(h.q, h.scale), undo(wq, ws, True), 2.0 ** -8)
    near(dh, undo(gq, gs), undo(wtq, wts, True), 2.0 ** -8)
    near(dW, undo(gtq, gts), undo(htq, hts), 2.0 ** -23)
    want = _bwd64(dh.cpu(), x.cpu(), w.cpu(), h.mean.cpu(), h.rstd.cpu())
    _within(dw, want[1], 512 * U * (dh.double().cpu() * want[3]).abs().sum(0))


# ---- refusals ------------------------------------------------------------------------------------

def test_refusals(ctx):
    from paper_2608_02611_b200 import binding
    L, E = binding.load(), binding.KbError
    x = torch.ones(4, 256, dtype=torch.bfloat16, device=DEV)
    w = torch.ones(256, device=DEV)
    q, s = ctx.quantize_blocks(x)
    for call in (lambda: ctx.quantize_blocks(x.to(torch.int32)), lambda: ctx.quantize_blocks(x, torch.float16),
                 lambda: ctx.quantize_blocks(x.cpu()), lambda: ctx.quantize_blocks(x.t()),
                 lambda: ctx.layernorm(x, w[:8]), lambda: ctx.layernorm(x, w.half()), lambda: ctx.layernorm(x, w, eps=0.0),
                 lambda: ctx.layernorm(x, w, eps=float("nan")), lambda: ctx.layernorm(x, w, quantize=torch.bfloat16),
                 lambda: ctx.layernorm(x, w, want_y=False, want_stats=False), lambda: ctx.layernorm(x.t(), None),
                 lambda: ctx.layernorm_backward(x.float(), x, w, w[:4], w[:4]),
                 lambda: ctx.layernorm_backward(x, x, w, w[:3], w[:4]),
                 lambda: ctx.matmul_blocks(q, s, q[:, :128], s), lambda: ctx.matmul_blocks(x, s, q, s),
                 lambda: ctx.matmul_blocks(q, s[:1], q, s), lambda: ctx.matmul_blocks(q, s, q, s.t().contiguous()),
                 lambda: ctx.matmul_blocks(q, s, q, s, out_dtype=torch.int32),
                 lambda: ctx.matmul_blocks(q, s, q, s, out=torch.empty(3, 4, device=DEV)),
                 lambda: ctx.matmul_blocks(q[:, :200][:, 8:], s, q[:, 8:200], s)):
        with pytest.raises(E):
            call()
    held = torch.full((4, 300), 5.0, device=DEV)
    st = torch.cuda.current_stream().cuda_stream
    BF, E4, F32 = binding.KB_BF16, binding.KB_F8E4M3, binding.KB_F32

    def mm(a=q.data_ptr(), lda=256, mode=0, M=4, N=4, K=256, d=held.data_ptr(), ldd=300, sa=s.data_ptr(), code=E4):
        return L.kb_matmul_blocks(ctx._h, a, lda, code, sa, q.data_ptr(), 256, E4, s.data_ptr(), mode, M, N, K, d, ldd, F32, st)

    assert mm(a=None) == 1 and mm(d=None) == 1 and mm(sa=None) == 1 and mm(ldd=3) == 1 and mm(lda=128) == 1
    assert mm(M=1 << 31) == 1 and mm(mode=2) == 3 and mm(code=BF) == 3
    assert mm(lda=257) == 2 and mm(a=q.data_ptr() + 1) == 2 and mm(d=held.data_ptr() + 2) == 2 and mm(sa=s.data_ptr() + 2) == 2
    assert b"16-byte" in L.kb_last_error(ctx._h) or b"aligned" in L.kb_last_error(ctx._h)
    assert L.kb_quantize_blocks(ctx._h, x.data_ptr(), 4, 256, 100, BF, 0, 0, q.data_ptr(), 256, E4, s.data_ptr(), st) == 1
    assert L.kb_quantize_blocks(ctx._h, x.data_ptr() + 1, 4, 256, 256, BF, 0, 0, q.data_ptr(), 256, E4, s.data_ptr(), st) == 2
    assert L.kb_quantize_blocks(ctx._h, x.data_ptr(), 4, 256, 256, BF, 2, 0, q.data_ptr(), 256, E4, s.data_ptr(), st) == 1
    assert L.kb_quantize_blocks(ctx._h, x.data_ptr(), 4, 256, 256, BF, 0, 0, q.data_ptr(), 256, E4, None, st) == 1
    assert L.kb_layernorm(ctx._h, x.data_ptr(), 4, 0, 256, BF, None, None, BF, 1e-5, x.data_ptr(), 256, None, None, None, 0, E4, None, st) == 1
    assert L.kb_layernorm(ctx._h, x.data_ptr(), 4, 256, 256, BF, None, None, BF, 1e-5, None, 0, None, None, q.data_ptr(), 256, E4, None, st) == 1
    assert L.kb_layernorm(None, x.data_ptr(), 4, 256, 256, BF, None, None, BF, 1e-5, None, 0, None, None, None, 0, E4, None, st) == 1
    torch.cuda.synchronize()
    assert bool((held == 5.0).all())       # nothing was launched
    assert ctx.poll() == 0


def test_workspace_refusal_leaves_the_context_usable():
    from paper_2608_02611_b200 import binding
    c = binding.Context(0)
    x = torch.randn(8, 512, device=DEV)
    m, r = torch.zeros(8, device=DEV), torch.ones(8, device=DEV)
    c.fail_next_allocs(1)
    with pytest.raises(binding.KbError) as e:
        c.layernorm_backward(x, x, None, m, r)
    assert e.value.status == 4
    dx, dw, db = c.layernorm_backward(x, x, None, m, r)
    _within(db, x.double().sum(0), 64 * U * x.double().abs().sum(0))
    c.close()
