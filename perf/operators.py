"""Timed cases of the model operators: layer norm, block quantisation, the 8-bit product.

A user of the gate who searches kernels for the linear layers of a model in 8-bit floating point
runs these next to it: they make the reference outputs, the operands and the baseline kernels that
candidates are compared with.  ``listed()`` names the cases, ``draw`` makes more of the same
ranges, ``prepare`` makes inputs from a seed, and ``run`` makes one pass: with ``own`` false in
elementary torch operations in 32 bits, with ``own`` true through the library.  ``exact`` gives the
outputs from the definition in 64 bits.

Layouts: matrices are row-major; 8-bit matrices have rows padded to 16 bytes; the scales of a
matrix [R][C] quantised in 1x128 blocks are [ceil(C/128)][R], in 128x128 tiles
[ceil(C/128)][ceil(R/128)].
"""
import math

import torch

own = False

BLOCK = 128
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
FP8_MAX = {"e4m3": 448.0, "e5m2": 57344.0}
EPS = 1e-5


# ---- the cases ---------------------------------------------------------------------------

def _norm(name, rows, cols, dtype, y, q):
    return {"name": name, "op": "layernorm", "rows": rows, "cols": cols, "dtype": dtype, "y": y, "q": q}


def _norm_bwd(name, rows, cols, dtype):
    return {"name": name, "op": "layernorm_backward", "rows": rows, "cols": cols, "dtype": dtype}


def _quant(name, rows, cols, dtype, fp8, tiles, transpose):
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "dtype": dtype, "fp8": fp8,
            "tiles": tiles, "transpose": transpose}


def _mm(name, M, N, K, out, a="e4m3", b="e4m3", tiles=True):
    return {"name": name, "op": "matmul", "M": M, "N": N, "K": K, "out": out, "a": a, "b": b, "tiles": tiles}


def listed():
    return [
        # serving: the norm of one token's hidden state, handed to the next product in 8 bits
        _norm("norm_1x8192_q", 1, 8192, "bf16", False, True),
        # training: a batch of tokens; y is kept for the weight's gradient, q feeds the product
        _norm("norm_16384x4096_yq", 16384, 4096, "bf16", True, True),
        # an fp32 model with odd sizes and no 8-bit consumer
        _norm("norm_4099x1001_fp32", 4099, 1001, "fp32", True, False),
        # training: the gradient of the norm of the largest hidden size and batch here
        _norm_bwd("norm_bwd_8192x8192", 8192, 8192, "bf16"),
        # a ragged batch in fp16
        _norm_bwd("norm_bwd_777x5003_fp16", 777, 5003, "fp16"),
        # gradients of a step, quantised along the tokens for the weight's gradient
        _quant("quant_4096x8192_T", 4096, 8192, "bf16", "e5m2", False, True),
        # weights after an update, quantised in tiles
        _quant("quant_8192x8192_tiles", 8192, 8192, "bf16", "e4m3", True, False),
        # serving: one token through a linear layer: the weights' bytes are the work
        _mm("mm_1x8192x8192", 1, 8192, 8192, "bf16"),
        # serving: a batch of streams through an odd-sized layer
        _mm("mm_48x5000x4100_fp16", 48, 5000, 4100, "fp16"),
        # a linear layer over a batch of 512 rows
        _mm("mm_512x8192x8192", 512, 8192, 8192, "bf16"),
        # the weight's gradient: both operands quantised along the tokens, fp32 out
        _mm("mm_dw_4096x4096x4096", 4096, 4096, 4096, "fp32", a="e5m2", tiles=False),
        # the largest product: a training batch
        _mm("mm_8192x8192x8192", 8192, 8192, 8192, "bf16"),
    ]


def _log(rng, lo, hi):
    """Log-uniform whole number; every second one is rounded to a multiple of 16."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and v >= 32:
        v = v // 16 * 16
    return min(max(v, lo), hi)


def draw(rng):
    op = rng.choice(["layernorm", "layernorm_backward", "quantize", "matmul", "matmul"])
    if op == "matmul":
        while True:
            M, N, K = _log(rng, 1, 8192), _log(rng, 64, 16384), _log(rng, 64, 16384)
            if M * N * K <= 8192 ** 3 and N * K <= 1 << 27 and 3072 not in (M, N, K):
                break
        tiles = rng.random() < 0.7
        c = _mm("", M, N, K, rng.choice(["bf16", "bf16", "fp16", "fp32"]), tiles=tiles,
                a=rng.choice(["e4m3", "e4m3", "e5m2"]), b="e4m3")
    else:
        while True:
            rows, cols = _log(rng, 1, 32768), _log(rng, 64, 20000)
            if rows * cols <= 1 << 26 and 3072 not in (rows, cols):
                break
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        if op == "layernorm":
            y, q = rng.choice([(True, False), (True, True), (False, True)])
            c = _norm("", rows, cols, dtype, y, q)
        elif op == "layernorm_backward":
            c = _norm_bwd("", rows, cols, dtype)
        else:
            c = _quant("", rows, cols, dtype, rng.choice(["e4m3", "e5m2"]), rng.random() < 0.5, rng.random() < 0.5)
    del c["name"]
    return c


# ---- inputs ------------------------------------------------------------------------------

def _hidden(gen, rows, cols, dtype):
    """Hidden states: each row with a mean of its own, each channel with a scale of its own, a few
    channels much larger than the rest."""
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    chan = torch.exp(0.5 * torch.randn(cols, generator=gen, device="cuda"))
    chan = torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.002, 20.0 * chan, chan)
    x.mul_(chan).add_(0.5 + torch.randn(rows, 1, generator=gen, device="cuda"))
    return x.to(dtype)


def _gradient(gen, rows, cols, dtype):
    """Gradients: small, and of a size that differs from token to token by a factor of a few."""
    g = torch.randn(rows, cols, generator=gen, device="cuda")
    g.mul_(0.01 * torch.exp(torch.randn(rows, 1, generator=gen, device="cuda"))).add_(0.002)
    return g.to(dtype)


def _padded(q):
    """A row-major 8-bit matrix whose rows start on 16-byte boundaries."""
    rows, cols = q.shape
    ld = (cols + 15) // 16 * 16
    held = torch.zeros(rows, ld, dtype=torch.uint8, device=q.device)
    held[:, :cols] = q.view(torch.uint8)
    return held.view(q.dtype)[:, :cols]


_handle = None


def _context():
    """The library's handle, one for the process as a user's program keeps it."""
    global _handle
    if _handle is None:
        from paper_2608_02611_b200 import binding
        _handle = binding.Context(torch.cuda.current_device())
    return _handle


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1000003 + 17)
    op = case["op"]
    s = dict(case)
    if op == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        x = _hidden(gen, M, K, torch.bfloat16) if case["tiles"] else _gradient(gen, M, K, torch.bfloat16)
        w = 0.02 * torch.randn(N, K, generator=gen, device="cuda") if case["tiles"] else _hidden(gen, N, K, torch.bfloat16)
        a, s["a_scale"] = _quantize_plain(x, case["a"], False, False)
        b, s["b_scale"] = _quantize_plain(w, case["b"], case["tiles"], False)
        s["a_q"], s["b_q"] = _padded(a), _padded(b)
        return s
    rows, cols, dtype = case["rows"], case["cols"], TYPES[case["dtype"]]
    if op == "quantize":
        if case["tiles"]:
            s["x"] = (0.02 * torch.randn(rows, cols, generator=gen, device="cuda")).to(dtype)
        else:
            s["x"] = _gradient(gen, rows, cols, dtype)
        return s
    s["x"] = _hidden(gen, rows, cols, dtype)
    s["weight"] = (1.0 + 0.1 * torch.randn(cols, generator=gen, device="cuda")).to(dtype)
    if op == "layernorm":
        s["bias"] = (0.1 * torch.randn(cols, generator=gen, device="cuda")).to(dtype)
        return s
    s["dy"] = _gradient(gen, rows, cols, dtype)
    x = s["x"].float()
    s["mean"] = x.mean(1)
    s["rstd"] = torch.rsqrt((x - s["mean"][:, None]).square().mean(1) + EPS)
    return s


# ---- the plain forms: elementary torch operations in 32 bits --------------------------------

def _fit(x, rows, cols):
    """x with zeros below and to the right, up to rows x cols."""
    if x.shape == (rows, cols):
        return x
    out = torch.zeros(rows, cols, dtype=x.dtype, device=x.device)
    out[:x.shape[0], :x.shape[1]] = x
    return out


def _quantize_plain(x, fp8, tiles, transpose):
    top = FP8_MAX[fp8]
    x = x.float()
    if transpose:
        x = x.t().contiguous()
    rows, cols = x.shape
    kb = -(-cols // BLOCK)
    rb = -(-rows // BLOCK)
    if tiles:
        v = _fit(x, rb * BLOCK, kb * BLOCK).view(rb, BLOCK, kb, BLOCK)
        amax = v.abs().amax((1, 3), keepdim=True)
    else:
        v = _fit(x, rows, kb * BLOCK).view(rows, 1, kb, BLOCK)
        amax = v.abs().amax((1, 3), keepdim=True)
    amax = amax.clamp_min(2.0 ** -100)
    q = (v * (top / amax)).clamp(-top, top).view(-1, kb * BLOCK)[:rows, :cols].to(FP8[fp8])
    return q, (amax / top)[:, 0, :, 0].t().contiguous()


def _layernorm_plain(x, weight, bias):
    x = x.float()
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    rstd = torch.rsqrt((xc * xc).mean(1, keepdim=True) + EPS)
    return xc * rstd * weight.float() + bias.float(), mean[:, 0], rstd[:, 0]


def _layernorm_backward_plain(dy, x, weight, mean, rstd):
    dy32 = dy.float()
    xh = (x.float() - mean[:, None]) * rstd[:, None]
    g = dy32 * weight.float()
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx.to(x.dtype), (dy32 * xh).sum(0).to(weight.dtype), dy32.sum(0).to(weight.dtype)


def _spread(scale, rows, cols, tiles):
    """The scale of each element of a matrix [rows][cols]."""
    s = scale.t()
    if tiles:
        s = s.repeat_interleave(BLOCK, 0)[:rows]
    return s.repeat_interleave(BLOCK, 1)[:, :cols]


def _matmul_plain(a, a_scale, b, b_scale, tiles, out):
    a32 = a.float() * _spread(a_scale, *a.shape, False)
    b32 = b.float() * _spread(b_scale, *b.shape, tiles)
    return (a32 @ b32.t()).to(out)


# ---- one pass ------------------------------------------------------------------------------

def run(s):
    op = s["op"]
    if own:
        kb = _context()
        if op == "layernorm":
            r = kb.layernorm(s["x"], s["weight"], s["bias"], EPS, want_y=s["y"],
                             quantize=torch.float8_e4m3fn if s["q"] else None)
            return {"y": r.y, "mean": r.mean, "rstd": r.rstd, "q": r.q, "scale": r.scale}
        if op == "layernorm_backward":
            return kb.layernorm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"])
        if op == "quantize":
            return kb.quantize_blocks(s["x"], FP8[s["fp8"]], tiles=s["tiles"], transpose=s["transpose"])
        return kb.matmul_blocks(s["a_q"], s["a_scale"], s["b_q"], s["b_scale"], out_dtype=TYPES[s["out"]])
    if op == "layernorm":
        y, mean, rstd = _layernorm_plain(s["x"], s["weight"], s["bias"])
        q, scale = _quantize_plain(y, "e4m3", False, False) if s["q"] else (None, None)
        return {"y": y.to(s["x"].dtype) if s["y"] else None, "mean": mean, "rstd": rstd, "q": q, "scale": scale}
    if op == "layernorm_backward":
        return _layernorm_backward_plain(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"])
    if op == "quantize":
        return _quantize_plain(s["x"], s["fp8"], s["tiles"], s["transpose"])
    return _matmul_plain(s["a_q"], s["a_scale"], s["b_q"], s["b_scale"], s["tiles"], TYPES[s["out"]])


# ---- what a pass cannot do without -----------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        kb = -(-K // BLOCK)
        scales = kb * (M + (-(-N // BLOCK) if case["tiles"] else N))
        return {"bytes": M * K + N * K + 4 * scales + M * N * SIZE[case["out"]], "flops": 2 * M * N * K}
    rows, cols, e = case["rows"], case["cols"], SIZE[case["dtype"]]
    n = rows * cols
    if op == "layernorm":
        out = (n * e if case["y"] else 0) + ((n + 4 * rows * -(-cols // BLOCK)) if case["q"] else 0)
        return {"bytes": n * e + 2 * cols * e + out + 8 * rows, "flops": 8 * n}
    if op == "layernorm_backward":
        return {"bytes": 3 * n * e + 3 * cols * e + 8 * rows, "flops": 16 * n}
    r, c = (cols, rows) if case["transpose"] else (rows, cols)
    blocks = -(-c // BLOCK) * (-(-r // BLOCK) if case["tiles"] else r)
    return {"bytes": n * e + n + 4 * blocks, "flops": 4 * n}


# ---- from the definition, in 64 bits ---------------------------------------------------------

def _blocked_exact(v, fp8, tiles):
    """(codes, scales) of a matrix in 64 bits; the sizes are padded by index, not by copying."""
    top = FP8_MAX[fp8]
    rows, cols = v.shape
    kb = -(-cols // BLOCK)
    col_block = torch.arange(cols, device=v.device) // BLOCK
    row_amax = torch.zeros(rows, kb, dtype=torch.float64, device=v.device)
    row_amax.scatter_reduce_(1, col_block.expand(rows, cols), v.abs(), "amax")
    if tiles:
        rb = -(-rows // BLOCK)
        row_block = torch.arange(rows, device=v.device) // BLOCK
        amax = torch.zeros(rb, kb, dtype=torch.float64, device=v.device)
        amax.scatter_reduce_(0, row_block[:, None].expand(rows, kb), row_amax, "amax")
        each = amax[row_block]
    else:
        amax = each = row_amax
    scale = torch.maximum(each, torch.full_like(each, 2.0 ** -100)) / top
    # to the nearest value of the format: a whole number of its steps at the element's exponent
    bits, low = (3, -6) if fp8 == "e4m3" else (2, -14)
    t = v / scale[:, col_block]
    step = torch.exp2(torch.floor(torch.log2(t.abs().clamp_min(2.0 ** (low - 20)))).clamp_min(low) - bits)
    codes = (torch.round(t / step) * step).clamp(-top, top)
    held = torch.maximum(amax, torch.full_like(amax, 2.0 ** -100)) / top
    return codes, held.t().contiguous()


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        k = torch.arange(K, device="cuda") // BLOCK
        n = torch.arange(N, device="cuda") // (BLOCK if case["tiles"] else 1)
        a = s["a_q"].double() * s["a_scale"].double()[k].t()
        b = s["b_q"].double() * s["b_scale"].double()[k][:, n].t()
        return torch.einsum("mk,nk->mn", a, b)
    x = s["x"].double()
    if op == "quantize":
        return _blocked_exact(x.t().contiguous() if case["transpose"] else x, case["fp8"], case["tiles"])
    if op == "layernorm":
        var, mean = torch.var_mean(x, 1, unbiased=False)
        rstd = (var + EPS) ** -0.5
        y = torch.addcmul(s["bias"].double(), (x - mean[:, None]) * rstd[:, None], s["weight"].double())
        codes, scale = _blocked_exact(y, "e4m3", False) if case["q"] else (None, None)
        return {"y": y if case["y"] else None, "mean": mean, "rstd": rstd, "q": codes, "scale": scale}
    # the gradient by the chain rule through xh = (x - mean) rstd, term by term
    dy, w = s["dy"].double(), s["weight"].double()
    rstd = s["rstd"].double()[:, None]
    xh = (x - s["mean"].double()[:, None]) * rstd
    dxh = dy * w
    n = x.shape[1]
    dvar_term = torch.einsum("rc,rc->r", dxh, xh)[:, None] / n
    dmean_term = dxh.sum(1, keepdim=True) / n
    dx = (dxh - dmean_term - xh * dvar_term) * rstd
    return dx, torch.einsum("rc,rc->c", dy, xh), torch.einsum("rc->c", dy)
