"""Attention and the rotation of heads from their definitions in 64 bits, with bounds on what the library's
roundings can add, for the GPU tests.  Everything here runs on the CPU.

u = 2^-24 is half a step of binary32.  The bounds count roundings of the definitions in include/kb_attention.h:
a matrix instruction adds its products with at most 2 u per addition, one exponential is off by at most 4 u
beside its argument's error, a sum of n terms by n u of the sum of magnitudes.
"""
import math

import torch

U = 2.0 ** -24
HALF_ULP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


def rope(x, weight, eps, positions, inv_freq, interleaved):
    """(value, bound) of heads x [tokens, heads, dim]; weight None: 1; eps None: no norm; inv_freq None: not turned."""
    d = x.double().cpu()
    dim, dtype = d.shape[-1], x.dtype
    if eps is not None:
        d = d / (d.square().mean(-1, keepdim=True) + eps).sqrt()
        if weight is not None:
            d = d * weight.double().cpu()
    out, size = d.clone(), d.abs()
    far = torch.zeros(1, 1, 1, dtype=torch.float64)
    if inv_freq is not None and inv_freq.numel():
        f = inv_freq.cpu()
        n = f.numel()
        pos = positions.cpu().double()
        angle = (pos[:, None] * f)[:, None]
        far = (pos.abs() * 2.0 ** -50)[:, None, None] * float(f.abs().max().clamp_min(1))
        a, b = ((slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n)))
        x0, x1 = d[..., a], d[..., b]
        out[..., a] = x0 * angle.cos() - x1 * angle.sin()
        out[..., b] = x1 * angle.cos() + x0 * angle.sin()
        size = d.abs()
        both = x0.abs() + x1.abs()
        size[..., a], size[..., b] = both, both
    # norm: sum of squares in chains of 13, division, root and two products, 15 u; cosine and sine 4 u (argument
    # below an eighth of a turn rounded once, 2 units of a value below 1); two products and a sum 3 u
    bound = size * (22 * U + far) + out.abs() * HALF_ULP[dtype] + TINY[dtype]
    return out, bound


def attend(q, k, v, seen, scale, dtype):
    """One sequence: q [rows, heads, dim], k and v [keys, kv heads, dim] (any floating type), seen [rows, keys]
    -> out, its bound, lse, its bound."""
    q, k, v = (t.double().cpu() for t in (q, k, v))
    rows, hq, dim = q.shape
    keys, hkv = k.shape[0], k.shape[1]
    g = hq // hkv
    if rows == 0 or keys == 0:
        z = torch.zeros(rows, hq, dim, dtype=torch.float64)
        m = torch.full((rows, hq), -math.inf, dtype=torch.float64)
        return z, z + TINY[dtype], m, torch.zeros_like(m)
    kk, vv = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
    s = torch.einsum("rhd,khd->hrk", q, kk) * scale
    size = torch.einsum("rhd,khd->hrk", q.abs(), kk.abs()) * scale
    hidden = ~seen.expand(rows, keys)
    s.masked_fill_(hidden, -math.inf)
    size.masked_fill_(hidden, 0.0)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    e = (s - top).exp()
    total = e.sum(-1, keepdim=True)
    none = total == 0
    w = e / torch.where(none, torch.ones_like(total), total)
    vz = torch.where(vv.isfinite(), vv, torch.zeros_like(vv))       # callers keep non-finite values out of what is seen
    out = torch.einsum("hrk,khd->rhd", w, vz)
    sized = torch.einsum("hrk,khd->rhd", w, vz.abs())
    lse = (top + total.log())[..., 0].t()
    finite = torch.where(s.isfinite(), s, torch.zeros_like(s))
    # a score: dim additions of products (2 u each) and its scaling; the exponent: the reference's and its own rounding;
    # the exponential itself
    delta = (2 * dim * U * size + 4 * U * (finite.abs() + top.abs()) + 8 * U).amax(-1).t()     # [rows, heads]
    n = keys + 64                                                                         # additions, the joins' among them
    rel = 2 * delta + HALF_ULP[dtype] + 2 * n * U
    most = vz.abs().amax() if vz.numel() else torch.tensor(0.0)
    # binary16's smallest steps are 2^-24, and the largest p is 2^7 or more
    lost = keys * 2.0 ** -31 * most if dtype == torch.float16 else 0.0
    bound = rel[..., None] * sized + lost + out.abs() * HALF_ULP[dtype] + TINY[dtype]
    lse_bound = delta + n * U + 8 * U * lse.abs().nan_to_num(0.0, 0.0, 0.0)
    return out, bound, lse, lse_bound


def within(got, want, bound, what=""):
    got = got.double().cpu()
    fine = want.isfinite()
    assert bool((got[~fine] == want[~fine]).all()), f"{what}: infinities"
    err = (got - want).abs()[fine]
    b = bound.expand_as(want)[fine]
    ok = err <= b
    assert bool(ok.all()), f"{what}: {int((~ok).sum())} of {ok.numel()} beyond the bound, worst {float((err / b).nan_to_num(math.inf).max()):.3g} of it"
