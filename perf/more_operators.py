"""Timed cases of the attention operators: norm and rotation of heads, prompts, paged decoding.

A user of the gate who searches attention kernels runs these next to it: they make the reference
outputs and the baseline kernels that candidates are compared with, for the three steps that a
serving program takes through an attention block.  ``listed()`` names the cases, ``draw`` makes more
of the same ranges, ``prepare`` makes inputs from a seed, and ``run`` makes one pass: with ``own``
false in elementary torch operations in 32 bits, with ``own`` true through the library.  ``exact``
gives the outputs from the definition in 64 bits.

Layouts: queries, keys and values of packed sequences are [tokens][heads][dim], slices of one matrix
[tokens][(q heads + 2 kv heads) dim] as a projection writes it; a cache is [pages][page][kv heads][dim].
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-6
THETA = 1e4


# ---- the cases ---------------------------------------------------------------------------

def _rope(name, lens, hq, hkv, dim, rot, dtype, interleaved=False, cache="none", page=64, far=0):
    """`far`: positions before the prompts' first tokens.  `cache`: "none", "both" (the rotated keys come
    back and go to the cache with the values) or "only" (they go to the cache alone)."""
    return {"name": name, "op": "qk_norm_rope", "lens": lens, "hq": hq, "hkv": hkv, "dim": dim, "rot": rot,
            "dtype": dtype, "interleaved": interleaved, "cache": cache, "page": page, "far": far}


def _prompt(name, lens, hq, hkv, dim, dtype, klens="", causal=True):
    """`lens` tokens per sequence ("2048*8": eight of 2048); `klens`: keys per sequence where there are more."""
    return {"name": name, "op": "attention", "lens": lens, "klens": klens, "hq": hq, "hkv": hkv, "dim": dim,
            "dtype": dtype, "causal": causal}


def _decode(name, lens, hq, hkv, dim, dtype, page):
    return {"name": name, "op": "attention_paged", "lens": lens, "hq": hq, "hkv": hkv, "dim": dim, "dtype": dtype,
            "page": page}


def _ragged(seed, n, lo, hi):
    """n lengths, log-uniform in [lo, hi], the longest among them, as a text."""
    rng = random.Random(seed)
    v = [hi] + [int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))) for _ in range(n - 1)]
    rng.shuffle(v)
    return ",".join(map(str, v))


def listed():
    return [
        # serving: one new token of one stream, far into a long text; its key and value go to the cache
        _rope("rope_1_to_cache", "1", 32, 8, 128, 128, "bf16", cache="only", far=100000),
        # prompts of a batch, normalised and rotated in one pass and stored for decoding
        _rope("rope_16384_both", "2048*8", 32, 8, 128, 128, "bf16", cache="both"),
        # a model in fp32 with small odd heads of which part is rotated, in neighbouring pairs, no cache
        _rope("rope_1001_fp32", "1001", 20, 5, 80, 32, "fp32", interleaved=True),
        # the smallest prompt: one question to a small model
        _prompt("prompt_77", "77", 8, 8, 64, "fp16"),
        # the attention output that the gate's third workload is modelled on: 8 x 32 x 2048 x 128
        _prompt("prompt_8x2048", "2048*8", 32, 32, 128, "fp16"),
        # packed requests of very different lengths
        _prompt("prompt_ragged", "1,17,130,511,1024,2000,4097,333,64,1280,255,3,700", 32, 8, 128, "bf16"),
        # the next piece of two long prompts whose first parts are there already; odd groups of heads
        _prompt("prompt_chunk", "512,300", 40, 8, 128, "bf16", klens="8192,5001"),
        # one long document: the largest
        _prompt("prompt_16384", "16384", 32, 8, 128, "bf16"),
        # one stream of a chat over a middling history: latency and the join count
        _decode("decode_1x8192", "8192", 32, 8, 128, "bf16", 64),
        # a batch of streams of very different ages
        _decode("decode_64_ragged", _ragged(7, 64, 1, 16384), 32, 8, 128, "bf16", 64),
        # a small model without grouped heads, pages that are no power of two
        _decode("decode_7_odd", "900,1,0,1733,64,47,3001", 12, 12, 96, "fp16", 48),
        # a full server: the cache's bytes are the work
        _decode("decode_128x4096", "4096*128", 64, 8, 128, "bf16", 128),
    ]


def _log(rng, lo, hi):
    return min(max(int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))), lo), hi)


def draw(rng):
    op = rng.choice(["qk_norm_rope", "attention", "attention", "attention_paged", "attention_paged"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    dim = rng.choice([64, 64, 80, 96, 128, 128, 128])
    hkv = rng.choice([1, 2, 4, 5, 8, 8])
    hq = hkv * rng.choice([1, 2, 3, 4, 4, 5, 8])
    if op == "qk_norm_rope":
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        n = _log(rng, 1, 8)
        lens = ",".join(str(_log(rng, 1, 2048)) for _ in range(n))
        rot = rng.choice([dim, dim, dim // 2])
        c = _rope("", lens, hq, hkv, dim, rot, dtype, rng.random() < 0.3, rng.choice(["none", "both", "only"]),
                  rng.choice([16, 48, 64, 128]), rng.choice([0, 0, _log(rng, 1, 1000000)]))
    elif op == "attention":
        n = _log(rng, 1, 16)
        top = 8192 if n == 1 else 4096
        q = [_log(rng, 1, top) for _ in range(n)]
        k = [v + _log(rng, 1, 2048) for v in q] if rng.random() < 0.25 else q
        while n * hq * max(q) * max(k) > 1 << 32:      # what the padded plain form can hold in little time
            hq, hkv = hq // hkv, 1
            q, k, n = q[:-1] or [v // 2 for v in q], k[:-1] or [v // 2 for v in k], max(1, n - 1)
        c = _prompt("", ",".join(map(str, q)), hq, hkv, dim, dtype, "" if k is q or k == q else ",".join(map(str, k)),
                    rng.random() < 0.8)
    else:
        n = _log(rng, 1, 128)
        lens = [_log(rng, 1, 16384) for _ in range(n)]
        if rng.random() < 0.2:
            lens[0] = 0
        while n * max(lens) > 1 << 20:
            lens = [v // 2 for v in lens]
        c = _decode("", ",".join(map(str, lens)), hq, hkv, dim, dtype, rng.choice([16, 48, 64, 128]))
    del c["name"]
    return c


def _lens(text):
    out = []
    for part in text.split(","):
        length, _, count = part.partition("*")
        out += [int(length)] * int(count or 1)
    return out


# ---- inputs ------------------------------------------------------------------------------

def _heads(gen, tokens, heads, dim, dtype, scale=1.0):
    """Heads of a projection: channels of different sizes."""
    x = torch.randn(tokens, heads, dim, generator=gen, device="cuda")
    x.mul_(torch.exp(0.3 * torch.randn(heads, dim, generator=gen, device="cuda"))).mul_(scale)
    return x.to(dtype)


def _offsets(lens):
    return torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)


def _pages(gen, lens, page):
    """Pages of a cache with a few spare ones, dealt out in random order: (number, table, [n][most])."""
    need = [-(-v // page) for v in lens]
    most, total = max(1, max(need)), sum(need)
    order = torch.randperm(total + 4, generator=gen, device="cuda").to(torch.int32)
    held = torch.arange(most, device="cuda")[None, :] < torch.tensor(need, device="cuda")[:, None]
    table = torch.zeros(len(lens), most, dtype=torch.int32, device="cuda")
    table[held] = order[:total]
    return total + 4, table


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
    gen.manual_seed(seed * 1000003 + 29)
    s = dict(case)
    dtype, hq, hkv, dim = TYPES[case["dtype"]], case["hq"], case["hkv"], case["dim"]
    lens = _lens(case["lens"])
    tokens = sum(lens)
    if case["op"] == "qk_norm_rope":
        qkv = _heads(gen, tokens, hq + 2 * hkv, dim, dtype, 2.0)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["q_weight"] = (1.0 + 0.2 * torch.randn(dim, generator=gen, device="cuda")).to(dtype)
        s["k_weight"] = (1.0 + 0.2 * torch.randn(dim, generator=gen, device="cuda")).to(dtype)
        s["inv_freq"] = THETA ** (-torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"])
        seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), torch.tensor(lens, device="cuda"))
        at = torch.arange(tokens, device="cuda") - _offsets(lens).long()[seq]
        s["positions"] = at + case["far"]
        if case["cache"] != "none":
            page = case["page"]
            pages, table = _pages(gen, lens, page)
            s["slots"] = table[seq, at // page].long() * page + at % page
            s["k_cache"] = _heads(gen, pages * page, hkv, dim, dtype).view(pages, page, hkv, dim)
            s["v_cache"] = _heads(gen, pages * page, hkv, dim, dtype).view(pages, page, hkv, dim)
        return s
    if case["op"] == "attention":
        klens = _lens(case["klens"]) if case["klens"] else lens
        s["q_offsets"], s["k_offsets"] = _offsets(lens), _offsets(klens)
        if klens == lens:                               # slices of one projection
            qkv = _heads(gen, tokens, hq + 2 * hkv, dim, dtype)
            s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        else:
            s["q"] = _heads(gen, tokens, hq, dim, dtype)
            s["k"], s["v"] = (_heads(gen, sum(klens), hkv, dim, dtype) for _ in range(2))
        return s
    s["q"] = _heads(gen, len(lens), hq, dim, dtype)
    pages, s["table"] = _pages(gen, lens, case["page"])
    s["lengths"] = torch.tensor(lens, device="cuda", dtype=torch.int32)
    s["k_cache"] = _heads(gen, pages * case["page"], hkv, dim, dtype).view(pages, case["page"], hkv, dim)
    s["v_cache"] = _heads(gen, pages * case["page"], hkv, dim, dtype).view(pages, case["page"], hkv, dim)
    return s


# ---- the plain forms: elementary torch operations in 32 bits --------------------------------

def _norm_rope_plain(x, weight, positions, inv_freq, rot, interleaved):
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    angle = positions.double()[:, None] * inv_freq      # 64 bits: a far position has few binary32 digits left
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _attend_plain(q, k, v, hidden):
    """q [n][kv heads][rows][dim], k and v [n][kv heads][keys][dim], `hidden` broadcasts to the scores."""
    score = (q / math.sqrt(q.shape[-1])) @ k.transpose(-1, -2)
    score.masked_fill_(hidden, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    weight = score.sub_(top).exp_()
    total = weight.sum(-1, keepdim=True)
    out = weight @ v / torch.where(total == 0, torch.ones_like(total), total)
    return out, (top + total.log())[..., 0]


def _padded(x, offsets, most):
    """Packed rows as [n][most][heads][dim] in 32 bits; what is past a sequence's end repeats some row."""
    at = (offsets[:-1, None].long() + torch.arange(most, device=x.device)).clamp_max(max(0, x.shape[0] - 1))
    return x[at].float()


def _prompt_plain(q, k, v, q_offsets, k_offsets, most_q, most_k, causal):
    hq, hkv, dim = q.shape[1], k.shape[1], q.shape[2]
    nq, nk = q_offsets.diff().long(), k_offsets.diff().long()
    n, g = nq.numel(), hq // hkv
    qp = _padded(q, q_offsets, most_q).view(n, most_q, hkv, g, dim).permute(0, 2, 3, 1, 4).reshape(n, hkv, g * most_q, dim)
    kp, vp = (_padded(t, k_offsets, most_k).transpose(1, 2) for t in (k, v))
    row, col = torch.arange(most_q, device=q.device), torch.arange(most_k, device=q.device)
    hidden = (col >= nk[:, None])[:, None, :]
    if causal:
        hidden = hidden | (col > row[:, None] + (nk - nq)[:, None, None])
    hidden = hidden.expand(n, most_q, most_k)[:, None].repeat(1, 1, g, 1)
    out, lse = _attend_plain(qp, kp, vp, hidden)
    seq = torch.repeat_interleave(torch.arange(n, device=q.device), nq, output_size=q.shape[0])
    at = torch.arange(q.shape[0], device=q.device) - q_offsets[seq].long()
    out = out.view(n, hq, most_q, dim)[seq, :, at]
    return out.to(q.dtype), lse.view(n, hq, most_q)[seq, :, at]


def _decode_plain(q, k_cache, v_cache, table, lengths):
    n, hq, dim = q.shape
    hkv = k_cache.shape[2]
    k, v = (t[table.long()].flatten(1, 2).transpose(1, 2).float() for t in (k_cache, v_cache))
    hidden = (torch.arange(k.shape[2], device=q.device) >= lengths[:, None])[:, None, None, :]
    out, lse = _attend_plain(q.float().view(n, hkv, hq // hkv, dim), k, v, hidden)
    return out.view(n, hq, dim).to(q.dtype), lse.view(n, hq)


# ---- one pass ------------------------------------------------------------------------------

def run(s):
    op = s["op"]
    if op == "qk_norm_rope":
        cached = s["cache"] != "none"
        if own:
            store = {"v": s["v"], "k_cache": s["k_cache"], "v_cache": s["v_cache"], "slots": s["slots"]} if cached else {}
            q, k = _context().qk_norm_rope(s["q"], s["k"], s["positions"], s["inv_freq"], s["q_weight"], s["k_weight"], EPS,
                                           interleaved=s["interleaved"], want_k=s["cache"] != "only", **store)
        else:
            q, k = (_norm_rope_plain(s[x], s[x + "_weight"], s["positions"], s["inv_freq"], s["rot"],
                                     s["interleaved"]).to(s[x].dtype) for x in ("q", "k"))
            if cached:
                s["k_cache"].flatten(0, 1)[s["slots"]] = k
                s["v_cache"].flatten(0, 1)[s["slots"]] = s["v"]
        return {"q": q, "k": k if s["cache"] != "only" else None, "k_cache": s["k_cache"] if cached else None,
                "v_cache": s["v_cache"] if cached else None}
    if op == "attention":
        if own:
            r = _context().attention(s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"], causal=s["causal"], want_lse=True)
            return {"out": r.out, "lse": r.lse}
        lens = _lens(s["lens"])
        klens = _lens(s["klens"]) if s["klens"] else lens
        out, lse = _prompt_plain(s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"], max(lens), max(klens), s["causal"])
        return {"out": out, "lse": lse}
    if own:
        r = _context().attention_paged(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], want_lse=True)
        return {"out": r.out, "lse": r.lse}
    out, lse = _decode_plain(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"])
    return {"out": out, "lse": lse}


# ---- what a pass cannot do without -----------------------------------------------------------

def _pairs(nq, nk, causal):
    """Pairs of a query and a key it sees."""
    if not causal:
        return nq * nk
    first = nk - nq + 1                                 # keys of the first query
    skipped = max(0, min(nq, -first + 1))
    first, rows = first + skipped, nq - skipped
    return rows * first + rows * (rows - 1) // 2


def work(case):
    hq, hkv, dim, e = case["hq"], case["hkv"], case["dim"], SIZE[case["dtype"]]
    lens = _lens(case["lens"])
    tokens = sum(lens)
    if case["op"] == "qk_norm_rope":
        row = tokens * dim * e
        moved = 2 * hq + hkv + {"none": hkv, "both": 4 * hkv, "only": 3 * hkv}[case["cache"]]
        return {"bytes": row * moved + tokens * (16 if case["cache"] != "none" else 8) + 2 * dim * e + 4 * case["rot"],
                "flops": tokens * (hq + hkv) * (4 * dim + 3 * case["rot"])}
    if case["op"] == "attention":
        klens = _lens(case["klens"]) if case["klens"] else lens
        pairs = sum(_pairs(a, b, case["causal"]) for a, b in zip(lens, klens))
        return {"bytes": e * dim * (2 * tokens * hq + 2 * sum(klens) * hkv) + 4 * tokens * hq + 8 * (len(lens) + 1),
                "flops": 4 * pairs * hq * dim}
    pages = sum(-(-v // case["page"]) for v in lens)
    return {"bytes": 2 * tokens * hkv * dim * e + len(lens) * (2 * hq * dim * e + 4 * hq + 4) + 4 * pages,
            "flops": 4 * tokens * hq * dim}


# ---- from the definition, in 64 bits ---------------------------------------------------------

def _norm_rope_exact(x, weight, s):
    """Each pair as a complex number, turned by multiplying with exp(i angle)."""
    x, rot = x.double(), s["rot"]
    x = weight.double() * x / (x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt()
    angle = torch.einsum("t,i->ti", s["positions"].double(), s["inv_freq"])
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    head, out = x[..., :rot], x.clone()
    if s["interleaved"]:
        out[..., :rot] = torch.view_as_real(torch.view_as_complex(head.unflatten(-1, (-1, 2)).contiguous()) * turn).flatten(-2)
    else:
        z = torch.complex(head[..., :rot // 2].contiguous(), head[..., rot // 2:].contiguous()) * turn
        out[..., :rot // 2], out[..., rot // 2:rot] = z.real, z.imag
    return out


def _attend_exact(q, k, v, seen):
    """One sequence: q [rows][heads][dim], k and v [keys][kv heads][dim], seen [rows][keys]; head by head."""
    rows, hq, dim = q.shape
    out = torch.zeros(rows, hq, dim, dtype=torch.float64, device=q.device)
    lse = torch.full((rows, hq), -math.inf, dtype=torch.float64, device=q.device)
    if k.shape[0] == 0 or rows == 0:
        return out, lse
    some = seen.any(1)
    for h in range(hq):
        j = h // (hq // k.shape[1])
        score = torch.einsum("rd,kd->rk", q[:, h].double(), k[:, j].double()) * dim ** -0.5
        score.masked_fill_(~seen, -math.inf)
        lse[:, h] = torch.logsumexp(score, 1)
        weight = score.sub_(torch.where(some, lse[:, h], 0.0)[:, None]).exp_()
        out[:, h] = torch.einsum("rk,kd->rd", weight, v[:, j].double())
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "qk_norm_rope":
        q, k = (_norm_rope_exact(s[x], s[x + "_weight"], s) for x in ("q", "k"))
        caches = {"k_cache": None, "v_cache": None}
        if case["cache"] != "none":
            for name, rows in (("k_cache", k), ("v_cache", s["v"].double())):
                held = s[name].double()
                held.view(-1, *held.shape[2:]).index_copy_(0, s["slots"], rows)
                caches[name] = held
        return {"q": q, "k": k if case["cache"] != "only" else None, **caches}
    lens = _lens(case["lens"])
    outs, lses = [], []
    if case["op"] == "attention":
        klens = _lens(case["klens"]) if case["klens"] else lens
        q0 = k0 = 0
        for nq, nk in zip(lens, klens):
            for r0 in range(0, nq, 4096):               # rows at a time, for the memory
                rows = min(4096, nq - r0)
                row = torch.arange(r0, r0 + rows, device="cuda")[:, None] + nk - nq
                seen = torch.arange(nk, device="cuda") <= (row if case["causal"] else torch.full_like(row, nk))
                o, m = _attend_exact(s["q"][q0 + r0:q0 + r0 + rows], s["k"][k0:k0 + nk], s["v"][k0:k0 + nk], seen)
                outs.append(o)
                lses.append(m)
            q0, k0 = q0 + nq, k0 + nk
    else:
        for b, n in enumerate(lens):
            at = torch.arange(n, device="cuda")
            slot = s["table"][b, at // case["page"]].long() * case["page"] + at % case["page"]
            o, m = _attend_exact(s["q"][b:b + 1], s["k_cache"].flatten(0, 1)[slot], s["v_cache"].flatten(0, 1)[slot],
                                 torch.ones(1, n, dtype=torch.bool, device="cuda"))
            outs.append(o)
            lses.append(m)
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
