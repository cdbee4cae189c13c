"""An attention block as a server runs it, judged by the gate.

A prompt of several requests goes through the library's operators (norm and rotation of the heads, which store the
keys and values by pages, then attention over the packed prompts), new tokens follow one at a time from the paged cache,
and the question a kernel search asks of an attention kernel is put to some candidates: which of several ways to
compute it passes the correctness gate against the output in 64 bits, and which passing one is fastest?  Two of the
candidates carry a planted mistake.

    python examples/attention_block.py [--requests 8] [--tokens 512] [--heads 32] [--kv-heads 8] [--dim 128]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_02611_b200 import binding as kb   # noqa: E402

PAGE = 64


class Cache:
    """Keys and values by pages, and which pages belong to which request."""

    def __init__(self, requests, most, kv_heads, dim, device):
        each = -(-most // PAGE)
        order = torch.randperm(requests * each, device=device).to(torch.int32)
        self.table = order.view(requests, each)
        self.k, self.v = (torch.zeros(requests * each, PAGE, kv_heads, dim, dtype=torch.bfloat16, device=device) for _ in range(2))

    def slots(self, request, position):
        return self.table[request, position // PAGE].long() * PAGE + position % PAGE


def split(qkv, heads, kv_heads):
    return qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]


def prompt(ctx, qkv, heads, kv_heads, lens, weights, inv_freq, cache):
    """The first pass over packed prompts -> outputs [tokens, heads, dim] and what they were made of."""
    q, k, v = split(qkv, heads, kv_heads)
    offsets = torch.tensor([0] + lens, device=qkv.device).cumsum(0).to(torch.int32)
    request = torch.repeat_interleave(torch.arange(len(lens), device=qkv.device), torch.tensor(lens, device=qkv.device))
    position = torch.arange(qkv.shape[0], device=qkv.device) - offsets[request].long()
    q, k = ctx.qk_norm_rope(q, k, position, inv_freq, *weights, v=v, k_cache=cache.k, v_cache=cache.v,
                            slots=cache.slots(request, position))
    return ctx.attention(q, k, v, offsets, want_lse=True), (q, k, v, offsets)


def token(ctx, qkv, heads, kv_heads, lengths, weights, inv_freq, cache):
    """One new token per request, which sees `lengths` earlier ones and itself."""
    q, k, v = split(qkv, heads, kv_heads)
    request = torch.arange(qkv.shape[0], device=qkv.device)
    q, _ = ctx.qk_norm_rope(q, k, lengths, inv_freq, *weights, want_k=False, v=v, k_cache=cache.k, v_cache=cache.v,
                            slots=cache.slots(request, lengths))
    return ctx.attention_paged(q, cache.k, cache.v, cache.table, (lengths + 1).to(torch.int32))


def plain(q, k, v, offsets, dtype, scale=None, shift=0):
    """Attention request by request in torch."""
    out = torch.empty_like(q, dtype=torch.float32)
    group = q.shape[1] // k.shape[1]
    for a, b in zip(offsets[:-1].tolist(), offsets[1:].tolist()):
        qs, ks, vs = (t[a:b].transpose(0, 1).to(dtype) for t in (q, k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)))
        s = (qs * (q.shape[2] ** -0.5 if scale is None else scale)) @ ks.transpose(1, 2)
        s.masked_fill_(torch.ones(b - a, b - a, dtype=torch.bool, device=q.device).triu(1 + shift), float("-inf"))
        out[a:b] = (torch.softmax(s, -1) @ vs).transpose(0, 1).float()
    return out


def ways(ctx, parts):
    """name -> a function that computes the prompts' attention."""
    q, k, v, offsets = parts
    return {
        "the library": lambda: ctx.attention(q, k, v, offsets).out,
        "plain, 32 bits": lambda: plain(q, k, v, offsets, torch.float32).bfloat16(),
        "plain, 16 bits": lambda: plain(q, k, v, offsets, torch.bfloat16).bfloat16(),
        "wrong scale": lambda: plain(q, k, v, offsets, torch.float32, scale=1.0 / q.shape[2]).bfloat16(),
        "sees the next token": lambda: plain(q, k, v, offsets, torch.float32, shift=1).bfloat16(),
    }


def timings(fns, repeats):
    out = torch.empty(len(fns), repeats, device="cuda")
    for i, fn in enumerate(fns):
        fn()
        for r in range(repeats):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            fn()
            b.record()
            b.synchronize()
            out[i, r] = a.elapsed_time(b)
    return out


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--requests", type=int, default=8)
    ap.add_argument("--tokens", type=int, default=512, help="of the longest request")
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--new", type=int, default=4, help="tokens that follow the prompts")
    ap.add_argument("--repeats", type=int, default=9)
    args = ap.parse_args(argv)
    torch.manual_seed(0)
    dev = torch.device("cuda", 0)
    ctx = kb.Context(0)
    lens = [max(1, args.tokens * (i + 1) // args.requests) for i in range(args.requests)]
    rows = args.heads + 2 * args.kv_heads
    weights = [torch.rand(args.dim, device=dev).add(0.5).bfloat16() for _ in range(2)]
    inv_freq = 1e4 ** (-torch.arange(0, args.dim, 2, dtype=torch.float64, device=dev) / args.dim)
    cache = Cache(args.requests, max(lens) + args.new, args.kv_heads, args.dim, dev)
    first, parts = prompt(ctx, torch.randn(sum(lens), rows, args.dim, device=dev).bfloat16(), args.heads, args.kv_heads, lens, weights,
                          inv_freq, cache)
    lengths = torch.tensor(lens, device=dev)
    for i in range(args.new):
        step = token(ctx, torch.randn(args.requests, rows, args.dim, device=dev).bfloat16(), args.heads, args.kv_heads, lengths + i, weights,
                     inv_freq, cache)
    assert bool(first.out.isfinite().all()) and bool(step.out.isfinite().all())
    # the gate: every way's output against 64 bits
    fns = ways(ctx, parts)
    ref = plain(*parts, torch.float64).bfloat16().contiguous()
    outs = [fn().contiguous() for fn in fns.values()]
    records = kb.records(ctx.screen(ref, outs, atol=2e-2, rtol=2e-2))
    t = timings(list(fns.values()), args.repeats)
    median, _, _ = ctx.adjudicate(t)
    survivors, n = ctx.select(ctx.screen(ref, outs, 2e-2, 2e-2), median, kb.KB_SELECT_ERR_THEN_TIME, budget=len(outs))
    passing = []
    for i, name in enumerate(fns):
        print(f"{name:20s} {'passes' if records['pass'][i] else 'fails '}  largest error {records['max_abs_err'][i]:.3g}  "
              f"{float(median[i]) * 1e3:9.1f} us")
        if records["pass"][i]:
            passing.append((float(median[i]), name))
    print(f"{int(n.item())} of {len(outs)} survive; the fastest of them: {min(passing)[1]}")
    assert ctx.poll() == 0
    ctx.close()
    return {name: bool(records["pass"][i]) for i, name in enumerate(fns)}


if __name__ == "__main__":
    main()
