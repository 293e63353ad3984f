"""Attention of a program that answers: prompts of different lengths packed one behind the other, a paged cache of keys and values (in the
storage type or in 8 bits), and attention of new tokens over that cache.

A case is one call: causal attention over packed prompts, attention of a chunk of new tokens (often one) over the pages of every sequence,
writing the new tokens' keys and values into the pages, or reading them back.  Keys and values come as column blocks of one
[tokens, heads + 2 kv_heads, d_h] projection, as a layer with a packed weight makes them; pages of a sequence lie anywhere in the cache.

The plain form pads the sequences to the longest one and computes in 32 bits; an 8-bit row is held as e4m3 values times a power of two of
its own, which makes the codes and the values they stand for exact.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn


def listed():
    return [
        # a handful of short prompts in fp32, one of a single token: a small model that needs the 1e-4 parity of the fp32 path
        dict(name="packed_short_f32", op="packed", dtype="f32", seqs=5, kv_lo=1, kv_hi=96, heads=12, kv_heads=12, d_h=64, causal=True, mix=1),
        # a batch of prompts of a chat service, grouped heads
        dict(name="packed_ragged_bf16", op="packed", dtype="bf16", seqs=9, kv_lo=100, kv_hi=2048, heads=32, kv_heads=8, d_h=128, causal=True, mix=2),
        # two long documents, a key head for every query head (32 heads of 128, the layer of the benchmark)
        dict(name="packed_long_bf16", op="packed", dtype="bf16", seqs=2, kv_lo=8192, kv_hi=8192, heads=32, kv_heads=32, d_h=128, causal=True, mix=3),
        # one conversation, one token: latency
        dict(name="decode_one_bf16", op="paged", dtype="bf16", cache="same", seqs=1, new_lo=1, new_hi=1, kv_lo=500, kv_hi=500, heads=32, kv_heads=8,
             d_h=128, page=16, causal=True, mix=4),
        # a step of a busy server over an 8-bit cache
        dict(name="decode_batch_e4m3", op="paged", dtype="bf16", cache="e4m3", seqs=64, new_lo=1, new_hi=1, kv_lo=256, kv_hi=8192, heads=32, kv_heads=8,
             d_h=128, page=64, causal=True, mix=5),
        # a few very long conversations: the split along the keys carries it
        dict(name="decode_long_bf16", op="paged", dtype="bf16", cache="same", seqs=6, new_lo=1, new_hi=1, kv_lo=16384, kv_hi=65536, heads=32, kv_heads=8,
             d_h=128, page=128, causal=True, mix=6),
        # prompts fed in chunks behind what the cache holds already
        dict(name="chunk_bf16", op="paged", dtype="bf16", cache="same", seqs=4, new_lo=200, new_hi=512, kv_lo=3000, kv_hi=16384, heads=32, kv_heads=8,
             d_h=128, page=64, causal=True, mix=7),
        # drafted tokens and short chunks of a small fp32 model
        dict(name="chunk_f32", op="paged", dtype="f32", cache="same", seqs=3, new_lo=1, new_hi=70, kv_lo=100, kv_hi=2000, heads=12, kv_heads=4,
             d_h=64, page=16, causal=True, mix=8),
        # the new tokens of a step, quantised into their pages: latency
        dict(name="write_step_e4m3", op="write", dtype="bf16", cache="e4m3", seqs=64, new_lo=1, new_hi=1, kv_lo=256, kv_hi=4096, heads=32, kv_heads=8,
             d_h=128, page=64, mix=9),
        # whole prompts, quantised as they are written
        dict(name="write_prompts_e4m3", op="write", dtype="bf16", cache="e4m3", seqs=8, new_lo=1500, new_hi=8192, kv_lo=1500, kv_hi=8192, heads=32,
             kv_heads=8, d_h=128, page=64, mix=10),
        # prefixes of a small cache read back where no quantisation is wanted
        dict(name="read_short_bf16", op="read", dtype="bf16", cache="same", seqs=16, new_lo=1, new_hi=300, kv_lo=1, kv_hi=300, heads=12, kv_heads=12,
             d_h=64, page=16, mix=11),
        # long conversations read back from 8 bits
        dict(name="read_long_e4m3", op="read", dtype="bf16", cache="e4m3", seqs=8, new_lo=4000, new_hi=32768, kv_lo=4000, kv_hi=32768, heads=32, kv_heads=8,
             d_h=128, page=128, mix=12),
    ]


def _near(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["packed", "paged", "paged", "write", "read"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    d_h = rng.choice([64, 128, 128, 32, 80, 96, 256])
    kv_heads = rng.choice([1, 2, 3, 4, 8, 12])
    case = dict(op=op, dtype=dtype, heads=kv_heads * rng.choice([1, 1, 2, 3, 4, 7, 8]), kv_heads=kv_heads, d_h=d_h, mix=rng.randrange(1 << 20))
    if op == "packed":
        seqs = _near(rng, 1, 64)
        hi = _near(rng, 1, min(8192 // seqs if seqs > 4 else 4096, math.isqrt(10**12 // (2 * case["heads"] * d_h * seqs))))
        return dict(case, seqs=seqs, kv_lo=_near(rng, 1, hi), kv_hi=hi, causal=rng.random() < 0.8)
    case |= dict(cache=rng.choice(["same", "e4m3"]), page=rng.choice([1, 8, 16, 16, 32, 64, 64, 128, 256]))
    if op == "paged":
        seqs = _near(rng, 1, 128)
        new_hi = rng.choice([1, 1, _near(rng, 1, 8), _near(rng, 1, 512)])
        hi = _near(rng, new_hi, max(new_hi, 131072 // seqs if new_hi <= 8 else min(32768 // seqs, 10**12 // (4 * case["heads"] * d_h * new_hi * seqs))))
        return dict(case, seqs=seqs, new_lo=rng.choice([1, _near(rng, 1, new_hi)]), new_hi=new_hi, kv_lo=_near(rng, 1, hi), kv_hi=hi, causal=rng.random() < 0.8)
    seqs = _near(rng, 1, 200)
    hi = _near(rng, 1, max(1, 65536 // seqs))
    new_hi = rng.choice([1, _near(rng, 1, hi), hi])
    return dict(case, seqs=seqs, new_lo=_near(rng, 1, new_hi), new_hi=new_hi, kv_lo=_near(rng, 1, hi), kv_hi=hi)


def _lengths(case):
    """(length, new tokens) of every sequence: the case's own, whatever the seed; the first is the largest."""
    rng = random.Random(case["mix"])
    got = []
    for s in range(case["seqs"]):
        length = _near(rng, case["kv_lo"], case["kv_hi"]) if s else case["kv_hi"]
        if case["op"] == "packed":
            got.append((length, length))
        else:
            got.append((length, min(length, _near(rng, case["new_lo"], case["new_hi"]) if s else case["new_hi"])))
    return got


def _quantised(x):
    """Rows of x (last axis) as e4m3 codes and biased exponents: the smallest power of two that brings the row into ±448."""
    fine = torch.isfinite(x)
    top = torch.where(fine, x.abs(), 0.0).amax(-1)
    part, exp = torch.frexp(top)
    exp = torch.where(top > 0, exp - 9 + (part > 0.875), -127).clamp(-127, 127)
    scaled = torch.where(fine, torch.ldexp(x, -exp.unsqueeze(-1)), float("nan"))
    return scaled.to(E4M3), (exp + 127).to(torch.uint8)


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    t, d_h, heads, hk = DTYPES[case["dtype"]], case["d_h"], case["heads"], case["kv_heads"]
    lengths = _lengths(case)
    new = [n for _, n in lengths]
    tokens = sum(new)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    offsets = [0]
    for n in new:
        offsets.append(offsets[-1] + n)
    st = {"case": case, "offsets": ints(offsets), "max_new": max(new), "max_length": max(n for n, _ in lengths), "tokens": tokens}
    # queries that look for something: scores with a standard deviation of 2
    qkv = torch.randn((tokens, heads + 2 * hk, d_h), generator=gen, device="cuda")
    qkv[:, :heads] *= 2.0
    qkv = qkv.to(t)
    st["Q"], st["K"], st["V"] = qkv[:, :heads], qkv[:, heads:heads + hk], qkv[:, heads + hk:]
    if case["op"] in ("packed", "paged"):
        st["out"] = torch.zeros((tokens, heads, d_h), dtype=t, device="cuda")
    if case["op"] == "packed":
        return st
    page = case["page"]
    most = -(-st["max_length"] // page)
    held = [-(-n // page) for n, _ in lengths]
    n_pages = sum(held) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    # a row of page numbers for each sequence; -1 where it has none
    slot = torch.arange(most, device="cuda").unsqueeze(0)
    held_d = ints(held).unsqueeze(1)
    first = torch.cumsum(held_d, 0) - held_d
    st["table"] = torch.where(slot < held_d, order[(first + slot).clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous()
    st["length"] = ints([n for n, _ in lengths])
    shape = (n_pages, hk, page, d_h)
    for name in ("K", "V"):
        pages = torch.zeros(shape, device="cuda") if case["op"] == "write" else torch.randn(shape, generator=gen, device="cuda")
        if case["cache"] == "e4m3":
            st[name + "_pages"], st[name + "_scale"] = _quantised(pages)
        else:
            st[name + "_pages"], st[name + "_scale"] = pages.to(t), None
        del pages
    if case["op"] == "read":
        st["K_out"], st["V_out"] = (torch.zeros((tokens, hk, d_h), dtype=t, device="cuda") for _ in range(2))
    return st


def _places(st):
    """(sequence, index among its new tokens) of every token of the packed tensors."""
    at = torch.arange(st["tokens"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(st["offsets"][1:].contiguous(), at, right=True)
    return seq, at - st["offsets"][seq]


def _padded(x, st):
    """Rows of the packed x by sequence, in 32 bits: [sequences, most new tokens, heads, d_h]; rows past a sequence's end are some other row."""
    at = st["offsets"][:-1, None] + torch.arange(st["max_new"], device="cuda", dtype=torch.int32)
    return x[at.clamp(max=st["tokens"] - 1)].float()


def _attend(q, k, v, seen, scale):
    """q [s, n, heads, d], k and v [s, kv_heads, m, d], seen [s, n, m] -> [s, n, heads, d]; a row that sees nothing is zero."""
    s, n, heads, d = q.shape
    hk = k.shape[1]
    g = heads // hk
    q = (q * scale).view(s, n, hk, g, d).permute(0, 2, 3, 1, 4).reshape(s, hk, g * n, d)
    p = torch.matmul(q, k.transpose(2, 3).contiguous()).view(s, hk, g, n, -1)
    p.masked_fill_(~seen[:, None, None], float("-inf"))
    top = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(top == float("-inf"), 0.0, top)).exp_().view(s, hk, g * n, -1)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    return o.view(s, hk, g, n, d).permute(0, 3, 1, 2, 4).reshape(s, n, heads, d)


def _values(pages, scale):
    """What the pages hold, in 32 bits."""
    x = pages.float()
    return x if scale is None else torch.ldexp(x, scale.to(torch.int32).unsqueeze(-1) - 127)


def _gathered(pages, scale, st):
    """The pages of every sequence one behind the other: [sequences, kv_heads, positions, d_h] in 32 bits."""
    table = st["table"].clamp(min=0)
    x = _values(pages[table] if scale is None else pages.view(torch.uint8)[table].view(E4M3), None if scale is None else scale[table])
    return x.permute(0, 2, 1, 3, 4).reshape(x.shape[0], x.shape[2], -1, x.shape[4])


def _slots(st):
    """(page, slot in it) of every new token."""
    seq, i = _places(st)
    at = st["length"][seq] - (st["offsets"][seq + 1] - st["offsets"][seq]) + i
    page = st["case"]["page"]
    return st["table"][seq, at // page], at % page


def run(st):
    case = st["case"]
    op = case["op"]
    if own:
        import paper_2403_02352_amd as atp
        if op == "packed":
            return atp.attention_packed(st["Q"], st["K"], st["V"], st["offsets"], causal=case["causal"], out=st["out"])
        cache = atp.PagedCache(st["K_pages"], st["V_pages"], st["K_scale"], st["V_scale"])
        if op == "paged":
            return atp.attention_paged(st["Q"], cache, st["table"], st["length"], st["offsets"], causal=case["causal"], max_new=st["max_new"], out=st["out"])
        if op == "write":
            atp.cache_write(cache, st["K"], st["V"], st["table"], st["length"], st["offsets"])
            return [x for x in (st["K_pages"], st["V_pages"], st["K_scale"], st["V_scale"]) if x is not None]
        return atp.cache_read(cache, st["table"], st["length"], st["offsets"], out=(st["K_out"], st["V_out"]))
    if op in ("packed", "paged"):
        q = _padded(st["Q"], st)
        new = st["offsets"][1:] - st["offsets"][:-1]
        if op == "packed":
            k, v = (_padded(st[x], st).transpose(1, 2).contiguous() for x in "KV")
            length = new
        else:
            k, v = (_gathered(st[x + "_pages"], st[x + "_scale"], st) for x in "KV")
            length = st["length"]
        key = torch.arange(k.shape[2], device="cuda")
        seen = (key < length[:, None])[:, None].expand(-1, q.shape[1], -1)
        if case["causal"]:
            at = (length - new)[:, None] + torch.arange(q.shape[1], device="cuda")
            seen = seen & (key <= at[:, :, None])
        o = _attend(q, k, v, seen, 1.0 / math.sqrt(case["d_h"]))
        seq, i = _places(st)
        st["out"].copy_(o[seq, i])
        return st["out"]
    page, slot = _slots(st)
    if op == "write":
        got = []
        for x in "KV":
            pages, scale = st[x + "_pages"], st[x + "_scale"]
            if scale is None:
                pages[page, :, slot] = st[x]
            else:
                codes, exp = _quantised(st[x].float())
                pages.view(torch.uint8)[page, :, slot] = codes.view(torch.uint8)
                scale[page, :, slot] = exp
            got.append((pages, scale))
        return [g[0] for g in got] + [g[1] for g in got if g[1] is not None]
    for x in "KV":
        pages, scale = st[x + "_pages"], st[x + "_scale"]
        if scale is None:
            st[x + "_out"].copy_(pages[page, :, slot])
        else:
            st[x + "_out"].copy_(_values(pages.view(torch.uint8)[page, :, slot].view(E4M3), scale[page, :, slot]))
    return st["K_out"], st["V_out"]


def work(case):
    lengths = _lengths(case)
    d_h, heads, hk = case["d_h"], case["heads"], case["kv_heads"]
    es = 2 if case["dtype"] == "bf16" else 4
    new, held = sum(n for _, n in lengths), sum(n for n, _ in lengths)
    row = (d_h + 1 if case.get("cache") == "e4m3" else d_h * es) * hk * 2   # keys and values of a position in the cache
    if case["op"] in ("write", "read"):
        return {"bytes": new * (row + 2 * hk * d_h * es), "flops": 0}
    seen = sum(n * length - (n * (n - 1) // 2 if case["causal"] else 0) for length, n in lengths)
    kv = new * hk * d_h * es * 2 if case["op"] == "packed" else held * row
    return {"bytes": new * heads * d_h * es * 2 + kv, "flops": 4 * d_h * heads * seen}


def _row64(x):
    """Codes of rows of x in 64 bits: the nearest value of 1 sign, 4 exponent (bias 7) and 3 mantissa bits, ties to even, of x over its row's power of two."""
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 448.0).clamp(min=-127.0))
    e = torch.where(top > 448.0 * torch.exp2(e), e + 1, torch.where(top <= 448.0 * torch.exp2(e - 1), e - 1, e)).clamp(min=-127.0)
    x = x / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    st = prepare(case, seed)
    lengths = _lengths(case)
    heads, hk, page = case["heads"], case["kv_heads"], case.get("page")
    first = [0]
    for _, n in lengths:
        first.append(first[-1] + n)

    def held(x, s, h, length):
        """What the cache holds of one sequence and head, [length, d_h]."""
        pages = st["table"][s, :-(-length // page)].long()
        at = (pages * hk + h)
        v = st[x + "_pages"].view(-1, page, case["d_h"])
        if st[x + "_scale"] is None:
            return v[at].double().reshape(-1, case["d_h"])[:length]
        v = v.view(torch.uint8)[at].view(E4M3).float().double()
        return (v * torch.exp2(st[x + "_scale"].view(-1, page)[at].double() - 127.0).unsqueeze(-1)).reshape(-1, case["d_h"])[:length]

    if case["op"] in ("packed", "paged"):
        out = torch.zeros((st["tokens"], heads, case["d_h"]), dtype=torch.float64, device="cuda")
        for s, (length, n) in enumerate(lengths):
            rows = slice(first[s], first[s + 1])
            hide = torch.arange(length, device="cuda")[None] > torch.arange(length - n, length, device="cuda")[:, None]
            for h in range(hk):
                if case["op"] == "packed":
                    k, v = st["K"][rows, h].double(), st["V"][rows, h].double()
                else:
                    k, v = held("K", s, h, length), held("V", s, h, length)
                for j in range(h * (heads // hk), (h + 1) * (heads // hk)):
                    a = st["Q"][rows, j].double() @ k.T / math.sqrt(case["d_h"])
                    if case["causal"]:
                        a = a.masked_fill(hide, float("-inf"))
                    out[rows, j] = torch.softmax(a, -1) @ v
        return out
    if case["op"] == "read":
        got = []
        for x in "KV":
            out = torch.empty((st["tokens"], hk, case["d_h"]), dtype=torch.float64, device="cuda")
            for s, (length, n) in enumerate(lengths):
                for h in range(hk):
                    out[first[s]:first[s + 1], h] = held(x, s, h, length)[length - n:]
            got.append(out)
        return got
    got = []
    for x in "KV":
        out = st[x + "_pages"].float().double()
        rows = st[x].double()
        rows = _row64(rows) if case["cache"] == "e4m3" else rows
        for s, (length, n) in enumerate(lengths):
            at = torch.arange(length - n, length, device="cuda")
            out[st["table"][s, at // page].long(), :, at % page] = rows[first[s]:first[s + 1]]
        got.append(out)
    return got + [None, None] if case["cache"] == "e4m3" else got
