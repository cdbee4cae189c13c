"""A linear layer behind a layer norm in 8-bit floating point, judged by the gate.

One training step of the layer y = norm(x) W^T with the library's operators (the norm hands its
output over in 8 bits, the products run on block-quantised operands, the norm's backward pass ends
the chain), then the question a kernel search asks of such a layer: which of several ways to
compute it passes the correctness gate against the unquantised output, and which passing one is
fastest?  The candidates differ in what they quantise and how; two of them carry a planted mistake.

    python examples/eight_bit_layer.py [--tokens 2048] [--width 4096] [--out 4096]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_02611_b200 import binding as kb   # noqa: E402

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2


def train_step(ctx, x, norm_weight, norm_bias, W, dY):
    """Forward and backward pass of norm + linear layer in 8 bits: (y, gradients by name)."""
    h = ctx.layernorm(x, norm_weight, norm_bias, quantize=E4M3)          # y for dW, codes for the product
    w, ws = ctx.quantize_blocks(W, tiles=True)
    y = ctx.matmul_blocks(h.q, h.scale, w, ws)                           # y = norm(x) W^T
    wt, wts = ctx.quantize_blocks(W, tiles=True, transpose=True)
    g, gs = ctx.quantize_blocks(dY, E5M2)
    dh = ctx.matmul_blocks(g, gs, wt, wts)                               # dh = dY W
    gt, gts = ctx.quantize_blocks(dY, E5M2, transpose=True)
    ht, hts = ctx.quantize_blocks(h.y, transpose=True)
    dW = ctx.matmul_blocks(gt, gts, ht, hts, out_dtype=torch.float32)    # dW = dY^T norm(x)
    dx, dnw, dnb = ctx.layernorm_backward(dh, x, norm_weight, h.mean, h.rstd)
    return y, {"x": dx, "W": dW, "norm_weight": dnw, "norm_bias": dnb}


def ways(ctx, x, norm_weight, norm_bias, W):
    """name -> a function that computes the layer's output; weights are laid out once."""
    e4, e4s = ctx.quantize_blocks(W, tiles=True)
    r4, r4s = ctx.quantize_blocks(W)
    e5, e5s = ctx.quantize_blocks(W, E5M2, tiles=True)
    shifted = e4s.roll(1, 0)

    def hidden(fmt):
        h = ctx.layernorm(x, norm_weight, norm_bias, want_y=False, want_stats=False, quantize=fmt)
        return h.q, h.scale

    def one_scale():   # mistake: every block takes the first block's scale
        q, s = hidden(E4M3)
        return ctx.matmul_blocks(q, s[:1].expand_as(s).contiguous(), e4, e4s)

    return {
        "e4m3, weight tiles": lambda: ctx.matmul_blocks(*hidden(E4M3), e4, e4s),
        "e4m3, weight rows": lambda: ctx.matmul_blocks(*hidden(E4M3), r4, r4s),
        "e5m2 activations": lambda: ctx.matmul_blocks(*hidden(E5M2), e4, e4s),
        "e5m2 weights": lambda: ctx.matmul_blocks(*hidden(E4M3), e5, e5s),
        "mistake: weight scales one block off": lambda: ctx.matmul_blocks(*hidden(E4M3), e4, shifted),
        "mistake: one activation scale": one_scale,
    }


def timings(calls, repeats):
    """[ways][repeats] milliseconds by CUDA events."""
    out = torch.empty(len(calls), repeats)
    for k, call in enumerate(calls):
        for _ in range(3):
            call()
        marks = [(torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)) for _ in range(repeats)]
        for a, b in marks:
            a.record()
            call()
            b.record()
        torch.cuda.synchronize()
        out[k] = torch.tensor([a.elapsed_time(b) for a, b in marks])
    return out.cuda()


def main(tokens=2048, width=4096, out=4096, repeats=16, log=print):
    ctx = kb.Context(torch.cuda.current_device())
    gen = torch.Generator(device="cuda")
    gen.manual_seed(260802611)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    # hidden states with channels of very different sizes: blocks need scales of their own
    x = (randn(tokens, width) * torch.exp(randn(width))).bfloat16()
    nw, nb = (torch.exp(randn(width))).bfloat16(), (0.1 * randn(width)).bfloat16()
    W = (0.02 * randn(out, width) * torch.exp(0.5 * randn(1, width))).bfloat16()
    dY = (1e-3 * randn(tokens, out)).bfloat16()

    y, grads = train_step(ctx, x, nw, nb, W, dY)
    log(f"one step: y {tuple(y.shape)}, " + ", ".join(f"d{k} {tuple(v.shape)}" for k, v in grads.items()))

    x32 = x.float()
    xh = (x32 - x32.mean(1, keepdim=True)) * torch.rsqrt(x32.var(1, unbiased=False, keepdim=True) + 1e-5)
    reference = ((xh * nw.float() + nb.float()) @ W.float().t()).bfloat16()
    table = ways(ctx, x, nw, nb, W)
    outputs = [call() for call in table.values()]
    # 8-bit codes carry 3 (e4m3) or 2 (e5m2) fraction bits: an output is off by several per cent of the
    # outputs' root mean square, whatever its own size is, and the worst of millions by ten times that;
    # an operand gone wrong shows as errors of the outputs' own size and more
    size = float(reference.float().square().mean().sqrt())
    atol = size
    screened = ctx.screen(reference, outputs, atol, 0.0)
    median, iqr, _ = ctx.adjudicate(timings(list(table.values()), repeats))
    best, n = ctx.select(screened, median, kb.KB_SELECT_TIME, len(table))
    status = ctx.poll()
    records = kb.records(screened)
    for k, name in enumerate(table):
        r = records[k]
        log(f"{name:40s} {'pass' if r['pass'] else 'FAIL':4s}  mismatches {int(r['mismatch_count']):9d}  "
            f"largest error {float(r['max_abs_err']) / size:7.3f} of the outputs' size  {float(median[k]) * 1e3:8.1f} us")
    order = [list(table)[i] for i in best[:int(n)].tolist()]
    log("passing, fastest first: " + "; ".join(order))
    ctx.close()
    return status, {name: bool(records[k]["pass"]) for k, name in enumerate(table)}, grads, order


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--width", type=int, default=4096)
    ap.add_argument("--out", type=int, default=4096)
    a = ap.parse_args()
    sys.exit(main(a.tokens, a.width, a.out)[0])
