"""The operators that keep keys and values in a quantised cache and attend over it, as cases that can be timed and compared.

A cache holds the keys and values of one layer in pages: elements [page][head][token of the page][dim] in FP4 (E2M1, two in a
byte, the even one in the low half) or FP8 (E4M3), and an E8M0 scale byte s for every 32 elements of a token's head; an element
stands for its value times 2^(s-127).  These are the bytes that the codec stores as FP4 and FP8 tensors and as streams of scale
bytes.  A page table [sequence][place] says which pages hold a sequence's tokens, `lens` how many tokens it has, and `first`
where its rows begin in tensors whose rows are the last tokens of all sequences, one sequence after the other: of a sequence's n
rows, row j is that of the token at lens - n + j.

  append     keys and values of the sequences' last tokens into the cache: the least power of two that keeps a block of 32
             within the format, elements rounded to nearest even
  read       the sequences' last tokens out of the cache
  attention  softmax(scale Q K^T) V over the cache, query heads in groups that share a head of the cache; a row sees the tokens
             up to its own (causal), the last `window` of them where that is not 0, or all; the logarithm of the softmax's sum
             comes with it

Where ``own`` is false ``run`` is the plain form in elementary torch operations, else the library's calls.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEVICE = "cuda:0"
REAL = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
WIDTH = {"f32": 4, "bf16": 2, "f16": 2}
BITS = {"fp4": 4, "e4m3": 8}
TOP = {"fp4": 6.0, "e4m3": 448.0}
FORMAT_CODE = {"fp4": 3, "e4m3": 2}
MOST_SCORES = 32 * 2048 * (32768 + 2048)      # of the listed prompt: query heads x rows x tokens
MOST_CACHED = 64 * 8192 * 8 * 128             # of the listed batch: elements of the keys
SPARE_PAGES = 3
FP4 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def listed():
    return [
        # A decoding step of sixteen sequences writes one token each: latency.
        dict(name="append_decode", op="append", seqs=16, new=1, past=2000, ragged=True, kv_heads=8, dim=128, page=16, fmt="fp4", src="bf16", fused=True),
        # A long prompt's keys and values on their way into the cache, out of a fused projection's result.
        dict(name="append_prompt", op="append", seqs=1, new=16384, past=0, ragged=False, kv_heads=8, dim=128, page=64, fmt="fp4", src="bf16", fused=True),
        # Ragged prompts behind others' cached beginnings, small heads, from FP16.
        dict(name="append_ragged", op="append", seqs=7, new=1999, past=777, ragged=True, kv_heads=5, dim=64, page=32, fmt="e4m3", src="f16", fused=False),
        # Cached sequences are read back, for a program that goes on in BF16.
        dict(name="read_batch", op="read", seqs=16, new=4096, past=0, ragged=True, kv_heads=8, dim=128, page=16, fmt="fp4", src="bf16", fused=False),
        # The last tokens of a few sequences in FP32, to be looked at.
        dict(name="read_tail", op="read", seqs=3, new=129, past=1500, ragged=True, kv_heads=2, dim=64, page=128, fmt="e4m3", src="f32", fused=False),
        # One sequence's decoding step: latency.
        dict(name="attention_one", op="attention", seqs=1, new=1, past=4095, ragged=False, q_heads=32, kv_heads=8, dim=128, page=16, fmt="fp4", src="bf16", causal=True, window=0),
        # A decoding batch of ragged sequences: bound by the cache's bytes.
        dict(name="attention_batch", op="attention", seqs=64, new=1, past=8191, ragged=True, q_heads=32, kv_heads=8, dim=128, page=64, fmt="fp4", src="bf16", causal=True, window=0),
        # Two very long sequences.
        dict(name="attention_long", op="attention", seqs=2, new=1, past=131071, ragged=False, q_heads=64, kv_heads=8, dim=128, page=128, fmt="fp4", src="bf16", causal=True, window=0),
        # Small heads in FP8, a sliding window, a group of an odd size.
        dict(name="attention_window", op="attention", seqs=33, new=1, past=5001, ragged=True, q_heads=28, kv_heads=4, dim=64, page=32, fmt="e4m3", src="f16", causal=True, window=2049),
        # A few guessed tokens a sequence are looked at together.
        dict(name="attention_guessed", op="attention", seqs=16, new=5, past=6000, ragged=True, q_heads=32, kv_heads=8, dim=128, page=32, fmt="e4m3", src="bf16", causal=True, window=0),
        # A piece of a long prompt: bound by the matrix products.
        dict(name="attention_prompt", op="attention", seqs=1, new=2048, past=32768, ragged=False, q_heads=32, kv_heads=8, dim=128, page=64, fmt="fp4", src="bf16", causal=True, window=0),
        # Ragged prompts, single tokens between them, in FP16.
        dict(name="attention_ragged", op="attention", seqs=9, new=1003, past=1500, ragged=True, q_heads=15, kv_heads=5, dim=64, page=16, fmt="fp4", src="f16", causal=True, window=0),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, even over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.5)))))))


def draw(rng):
    op = rng.choice(["append", "read", "attention", "attention", "attention"])
    kv_heads, dim, page = rng.choice([1, 2, 3, 4, 5, 8, 8]), rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128])
    fmt, ragged = rng.choice(["fp4", "fp4", "e4m3"]), rng.random() < 0.7
    if op != "attention":
        new, seqs = _spread(rng, 1, 16384), _spread(rng, 1, 64)
        new = max(1, min(new, 16384 * 8 * 128 // (seqs * kv_heads * dim)))
        return dict(op=op, seqs=seqs, new=new, past=rng.choice([0, _spread(rng, 1, 2000)]), ragged=ragged, kv_heads=kv_heads, dim=dim, page=page, fmt=fmt,
                    src=rng.choice(["bf16", "bf16", "f16", "f32"]), fused=rng.random() < 0.5)
    group = rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 8, 16])
    new = rng.choice([1, 1, 1, _spread(rng, 2, 8), _spread(rng, 16, 2048)])
    seqs = _spread(rng, 1, 128)
    past = max(0, min(_spread(rng, 16, 131072), MOST_CACHED // (seqs * kv_heads * dim) - new, MOST_SCORES // (seqs * kv_heads * group * new) - new))
    causal = rng.random() < 0.9
    return dict(op=op, seqs=seqs, new=new, past=past, ragged=ragged, q_heads=kv_heads * group, kv_heads=kv_heads, dim=dim, page=page, fmt=fmt,
                src=rng.choice(["bf16", "bf16", "f16"]), causal=causal, window=_spread(rng, 16, 4096) if causal and rng.random() < 0.25 else 0)


def _ceil(a, b):
    return -(-a // b)


def _lengths(case):
    """(tokens of each sequence, rows of each sequence), for the sizes alone, so that outputs of all inputs have one shape."""
    r = random.Random(case["seqs"] + 1000 * case["new"] + 10 ** 8 * case["past"])
    some = lambda most, least: r.randint(max(least, most // 4), most) if case["ragged"] and most > least else most  # noqa: E731
    new = [some(case["new"], 1) for _ in range(case["seqs"])]
    return [some(case["past"], 0) + n for n in new], new


def _randn(shape, g):
    return torch.randn(shape, generator=g, device=DEVICE)


def _keys(shape, g):
    """Gaussian values with a few channels that stand out, as keys have them."""
    x = _randn(shape, g)
    return x.mul_(1.0 + 4.0 * (torch.rand(shape[-1], generator=g, device=DEVICE) < 0.05))


# ---- the plain form -----------------------------------------------------------------------------------------------------------

def _quantize(x, fmt):
    """(elements, scale bytes) of x[..., dim] in 32 bits."""
    x = x.float()
    xb = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    fraction, exponent = torch.frexp(xb.abs().amax(dim=-1, keepdim=True))
    top_fraction, top_exponent = math.frexp(TOP[fmt])
    e = exponent - top_exponent + (fraction > top_fraction).int()
    e = torch.where(fraction > 0, e, torch.full_like(e, -127)).clamp(-127, 127)
    y = torch.ldexp(xb, -e).reshape(x.shape)
    scales = (e + 127).to(torch.uint8).squeeze(-1)
    if fmt == "e4m3":
        return y.to(torch.float8_e4m3fn).view(torch.uint8), scales
    a = y.abs()
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = code + (torch.signbit(y).to(torch.uint8) << 3)
    return code[..., 0::2] | (code[..., 1::2] << 4), scales


def _values(elems, scales, fmt):
    """What the elements stand for, in 32 bits."""
    if fmt == "e4m3":
        v = elems.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor(FP4 + [-f for f in FP4], device=DEVICE)
        v = torch.stack((table[(elems & 15).int()], table[(elems >> 4).int()]), dim=-1).flatten(-2)
    s = torch.ldexp(torch.ones(scales.shape, device=DEVICE), scales.int() - 127)
    return (v.reshape(*scales.shape, 32) * s.unsqueeze(-1)).reshape(v.shape)


def _places(s):
    """(page, token of the page) of every row."""
    pos, seq = s["row_pos"], s["row_seq"]
    return s["page_table"][seq, pos // s["page"]].long(), pos % s["page"]


def _tokens(elems, scales, s):
    """All tokens of all sequences, [sequence][head][token][dim], in 32 bits; behind a sequence's last token are those of page 0."""
    take = lambda t: t[s["page_table"].long()].transpose(2, 3).flatten(1, 2).transpose(1, 2)  # noqa: E731
    return _values(take(elems).contiguous(), take(scales), s["fmt"])


def _attention(s):
    seqs, heads, group, dim, new = s["seqs"], s["kv_heads"], s["q_heads"] // s["kv_heads"], s["dim"], s["most_new"]
    q = torch.zeros((seqs, new, heads, group, dim), device=DEVICE)
    q[s["row_seq"], s["row_nr"]] = s["q"].float().reshape(-1, heads, group, dim)
    q = q.permute(0, 2, 3, 1, 4).reshape(seqs, heads, group * new, dim)
    x = torch.matmul(q, _tokens(s["k_elems"], s["k_scales"], s).transpose(-1, -2)) * s["scale"]
    token = torch.arange(x.shape[-1], device=DEVICE)
    lens, count = s["lens"].long(), (s["first"][1:] - s["first"][:-1]).long()
    pos = (lens - count).unsqueeze(1) + torch.arange(new, device=DEVICE)                       # [sequence][row]
    last = pos if s["causal"] else (lens - 1).unsqueeze(1).expand_as(pos)
    hidden = (token > last.unsqueeze(-1)) | (token >= lens.reshape(-1, 1, 1))
    if s["window"]:
        hidden = hidden | (token <= pos.unsqueeze(-1) - s["window"])
    x = x.reshape(seqs, heads, group, new, -1).masked_fill_(hidden.reshape(seqs, 1, 1, new, -1), -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    p = torch.exp(x.sub_(torch.where(top > -math.inf, top, torch.zeros_like(top))))
    total = p.sum(dim=-1, keepdim=True)
    y = torch.matmul(p.reshape(seqs, heads, group * new, -1), _tokens(s["v_elems"], s["v_scales"], s)).reshape(seqs, heads, group, new, dim)
    y = torch.where(total > 0, y / total, torch.zeros_like(y))
    lse = (top + torch.log(total)).squeeze(-1)
    at = (s["row_seq"], s["row_nr"])
    return [y.permute(0, 3, 1, 2, 4)[at].reshape(-1, s["q_heads"], dim).to(REAL[s["src"]]), lse.permute(0, 3, 1, 2)[at].reshape(-1, s["q_heads"])]


# ---- what the tools call ------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    s = dict(case)
    lens, new = _lengths(case)
    seqs, heads, dim, page, fmt, src = (s[n] for n in ("seqs", "kv_heads", "dim", "page", "fmt", "src"))
    places = max(_ceil(n, page) for n in lens)
    used = [_ceil(n, page) for n in lens]
    pages = sum(used) + SPARE_PAGES
    order = torch.randperm(pages, generator=g, device=DEVICE).int().tolist()
    table = torch.zeros((seqs, places), dtype=torch.int32)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = torch.tensor(order[at: at + n], dtype=torch.int32)
        at += n
    first = [0]
    for n in new:
        first.append(first[-1] + n)
    rows = first[-1]
    s["page_table"] = table.to(DEVICE)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEVICE)
    s["first"] = torch.tensor(first, dtype=torch.int32, device=DEVICE)
    s["row_seq"] = torch.repeat_interleave(torch.arange(seqs), torch.tensor(new)).to(DEVICE)
    s["row_nr"] = torch.arange(rows, device=DEVICE) - s["first"].long()[s["row_seq"]]
    s["row_pos"] = (s["lens"].long() - torch.tensor(new, device=DEVICE))[s["row_seq"]] + s["row_nr"]
    s["most_new"] = max(new)
    width = dim * BITS[fmt] // 8
    for name in ("k", "v"):
        s[name + "_elems"] = torch.zeros((pages, heads, page, width), dtype=torch.uint8, device=DEVICE)
        s[name + "_scales"] = torch.zeros((pages, heads, page, dim // 32), dtype=torch.uint8, device=DEVICE)
        if s["op"] != "append":
            some = 1 << 28
            step = max(1, some // (heads * page * dim))
            for i in range(0, pages, step):
                shape = (min(step, pages - i), heads, page, dim)
                s[name + "_elems"][i: i + step], s[name + "_scales"][i: i + step] = _quantize(_keys(shape, g) if name == "k" else _randn(shape, g), fmt)
    if s["op"] == "attention":
        s["scale"] = 1.0 / math.sqrt(dim)
        s["q"] = _randn((rows, s["q_heads"], dim), g).to(REAL[src])
    elif s["op"] == "append":
        if s["fused"]:                                           # slices of one projection's result, queries before them
            qkv = _keys((rows, 6, heads, dim), g).to(REAL[src])
            s["k"], s["v"] = qkv[:, 4], qkv[:, 5]
        else:
            s["k"], s["v"] = _keys((rows, heads, dim), g).to(REAL[src]), _randn((rows, heads, dim), g).to(REAL[src])
    if own:
        from paper_2508_19263_b200 import binding as zc
        s["cache"] = zc.KvCache(s["k_elems"], s["k_scales"], s["v_elems"], s["v_scales"], FORMAT_CODE[fmt])
        s["batch"] = zc.KvBatch(s["page_table"], s["lens"], s["first"], s["most_new"])
        if s["op"] == "attention":
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty((rows, s["q_heads"]), device=DEVICE)
            s["workspace"] = torch.empty(zc.kv_attention_workspace_bytes(s["cache"], s["batch"], s["q_heads"]), dtype=torch.uint8, device=DEVICE)
        elif s["op"] == "read":
            s["k"], s["v"] = (torch.empty((rows, heads, dim), dtype=REAL[src], device=DEVICE) for _ in range(2))
    return s


def _state(s):
    """The cache: FP8 elements and scales as their values, FP4 elements as they lie there, two in a byte."""
    seen = [t.view(torch.float8_e4m3fn) if s["fmt"] == "e4m3" else t for t in (s["k_elems"], s["v_elems"])]
    return seen + [t.view(torch.float8_e8m0fnu) for t in (s["k_scales"], s["v_scales"])]


def _run_own(s):
    from paper_2508_19263_b200 import binding as zc
    if s["op"] == "append":
        zc.kv_append(s["cache"], s["batch"], s["k"], s["v"])
        return _state(s)
    if s["op"] == "read":
        return list(zc.kv_read(s["cache"], s["batch"], s["k"], s["v"]))
    zc.kv_attention(s["cache"], s["batch"], s["q"], s["out"], s["workspace"], scale=s["scale"], causal=s["causal"], window=s["window"], d_lse=s["lse"])
    return [s["out"], s["lse"]]


def run(s):
    if own:
        return _run_own(s)
    if s["op"] == "attention":
        return _attention(s)
    page, place = _places(s)
    if s["op"] == "append":
        s["k_elems"][page, :, place], s["k_scales"][page, :, place] = _quantize(s["k"], s["fmt"])
        s["v_elems"][page, :, place], s["v_scales"][page, :, place] = _quantize(s["v"], s["fmt"])
        return _state(s)
    return [_values(s[n + "_elems"][page, :, place], s[n + "_scales"][page, :, place], s["fmt"]).to(REAL[s["src"]]) for n in ("k", "v")]


def work(case):
    c, token = case, 2 * case["kv_heads"] * (case["dim"] * BITS[case["fmt"]] // 8 + case["dim"] // 32)       # a token's bytes in the cache
    lens, new = _lengths(case)
    if c["op"] != "attention":
        return {"bytes": sum(new) * (token + 2 * c["kv_heads"] * c["dim"] * WIDTH[c["src"]]), "flops": 0}
    seen = read = 0
    for n, m in zip(lens, new):
        window = c["window"] or n
        seen += sum(min(window, p + 1) for p in range(n - m, n)) if c["causal"] else n * m
        read += min(n, window + m - 1)
    rows = sum(new) * c["q_heads"]
    return {"bytes": read * token + rows * (2 * c["dim"] * WIDTH[c["src"]] + 4), "flops": 4 * c["dim"] * c["q_heads"] * seen}


# ---- the operators once more, from their definition, in 64 bits -------------------------------------------------------------

def _decoded(fmt):
    """The values of the 256 bytes of E4M3, or of the 16 halves of a byte of FP4, from their sign, exponent and mantissa bits."""
    bits, bias, width = (3, 7, 8) if fmt == "e4m3" else (1, 1, 4)
    sign = 1 << (width - 1)
    values = []
    for code in range(2 * sign):
        e, f = (code & (sign - 1)) >> bits, code & ((1 << bits) - 1)
        v = math.ldexp(f, 1 - bias - bits) if e == 0 else math.ldexp(f + (1 << bits), e - bias - bits)
        if fmt == "e4m3" and code & 127 == 127:
            v = math.nan
        values.append(-v if code & sign else v)
    return torch.tensor(values, dtype=torch.float64, device=DEVICE)


def _one(elems, scales, fmt):
    """Values of rows of elements [.., bytes] with their scale bytes [.., blocks]."""
    table = _decoded(fmt)
    v = table[elems.long()] if fmt == "e4m3" else torch.stack((table[(elems % 16).long()], table[(elems // 16).long()]), -1).flatten(-2)
    return v * torch.exp2(scales.double() - 127.0).repeat_interleave(32, -1)


def _nearest(x, fmt):
    """(values, scales) by the definition: least power of two, then the nearest value, ties to the even one."""
    bits, least = (3, -6) if fmt == "e4m3" else (1, 0)
    x = x.double()
    amax = x.reshape(*x.shape[:-1], -1, 32).abs().amax(-1)
    e = torch.floor(torch.log2(amax.clamp(min=2.0 ** -200) / TOP[fmt])) - 1
    for _ in range(3):
        e = e + (torch.exp2(e) * TOP[fmt] < amax)
    e = torch.where(amax > 0, e.clamp(-127, 127), torch.full_like(e, -127.0))
    v = x / torch.exp2(e).repeat_interleave(32, -1)
    p = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -60)))
    p = p - (torch.exp2(p) > v.abs()).double() + (torch.exp2(p + 1) <= v.abs()).double()
    step = torch.exp2(p.clamp(min=least) - bits)
    return torch.round(v / step) * step, torch.exp2(e)


def exact(case, seed):
    s = prepare(case, seed)
    lens, new = _lengths(case)
    page, fmt, heads, dim = s["page"], s["fmt"], s["kv_heads"], s["dim"]
    table, first = s["page_table"].tolist(), s["first"].tolist()
    if s["op"] == "append":
        values, scales = [], []
        for name in ("k", "v"):
            nearest, scale = _nearest(s[name], fmt)
            pages = s[name + "_elems"].shape[:3]
            values.append(torch.zeros((*pages, dim), dtype=torch.float64, device=DEVICE))
            scales.append(torch.full((*pages, dim // 32), 2.0 ** -127, dtype=torch.float64, device=DEVICE))        # scale bytes of 0
            for b, n in enumerate(new):
                for j0 in range((lens[b] - n) // page * page, lens[b], page):        # the rows that fall into this page
                    lo, hi = max(j0, lens[b] - n), min(j0 + page, lens[b])
                    r = first[b] + lo - (lens[b] - n)
                    at = (table[b][j0 // page], slice(None), slice(lo - j0, hi - j0))
                    values[-1][at], scales[-1][at] = nearest[r: r + hi - lo].transpose(0, 1), scale[r: r + hi - lo].transpose(0, 1)
        return (values if fmt == "e4m3" else [None, None]) + scales       # bytes of FP4 are compared as they are
    gather = lambda t, b: torch.cat([t[i] for i in table[b][: _ceil(lens[b], page)]], dim=1)[:, : lens[b]]  # noqa: E731
    if s["op"] == "read":
        parts = [[_one(gather(s[n + "_elems"], b), gather(s[n + "_scales"], b), fmt)[:, lens[b] - new[b]:].transpose(0, 1) for b in range(s["seqs"])] for n in ("k", "v")]
        return [torch.cat(p) for p in parts]
    group = s["q_heads"] // heads
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEVICE)
    for b in range(s["seqs"]):
        k, v = (_one(gather(s[n + "_elems"], b), gather(s[n + "_scales"], b), fmt) for n in ("k", "v"))
        pos = torch.arange(lens[b] - new[b], lens[b], device=DEVICE).reshape(-1, 1)
        token = torch.arange(lens[b], device=DEVICE)
        seen = (token <= pos) if s["causal"] else torch.ones((new[b], lens[b]), dtype=torch.bool, device=DEVICE)
        if s["window"]:
            seen = seen & (token > pos - s["window"])
        rows = slice(first[b], first[b + 1])
        for h in range(s["q_heads"]):
            x = (s["q"][rows, h].double() @ k[h // group].t()) * s["scale"]
            x = torch.where(seen, x, torch.full_like(x, -math.inf))
            lse[rows, h] = torch.logsumexp(x, dim=1)
            out[rows, h] = torch.softmax(x, dim=1) @ v[h // group]
    return [out, lse]
