"""The operators that work on FP8 matrices with block scales, as cases that can be timed and compared.

A matrix is held as FP8 elements (E4M3 or E5M2, rows of a pitch that is a multiple of 16 bytes) and E8M0 scale bytes s,
one for each block of 128 columns and of 1 row or 128 rows; an element stands for its FP8 value times 2^(s-127).  These
are the bytes that the codec stores as FP8 tensors and as streams of scale bytes.

  quantize  a matrix in FP32, BF16 or FP16 into FP8 and scale bytes, the transposed matrix as well where asked for: the
            smallest power of two that keeps a block within the format, elements rounded to nearest even
  matmul    D = A B^T of two such matrices: a linear layer (A activations, B weights), the gradient of its input (A the
            output's gradient, B the transposed weights) and of its weights (both operands transposed, over the tokens)
  moe       a mixture-of-experts layer for a few tokens: router, softmax over the top_k largest logits (ties go to the
            lowest index), gated SiLU experts with FP8 weights in 128 x 128 blocks, weighted sum

Where ``own`` is false ``run`` is the plain form in elementary torch operations, else the library's calls.
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda:0"
FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
FORMAT_CODE = {"e4m3": 2, "e5m2": 5}
MANTISSA = {"e4m3": 3, "e5m2": 2}
BIAS = {"e4m3": 7, "e5m2": 15}
TOP = {"e4m3": 448.0, "e5m2": 57344.0}
REAL = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
WIDTH = {"f32": 4, "bf16": 2, "f16": 2}
MOST_FLOPS = 2 * 8192 * 14336 * 4096


def listed():
    return [
        # Activations of a decoding batch of sixteen sequences in front of a projection: latency.
        dict(name="quantize_decode", op="quantize", rows=16, cols=4096, src="bf16", fmt="e4m3", block=1, transposed=False),
        # A weight matrix of an 8B-shaped layer on its way into an FP8 checkpoint, from its FP32 master copy.
        dict(name="quantize_weight", op="quantize", rows=14336, cols=4096, src="f32", fmt="e4m3", block=128, transposed=False),
        # A gradient of a training step, needed along both axes: for the input's and for the weights' gradient.
        dict(name="quantize_grad_both", op="quantize", rows=8192, cols=4096, src="bf16", fmt="e5m2", block=1, transposed=True),
        # One sequence's ragged prompt, head count and width off every tile.
        dict(name="quantize_ragged", op="quantize", rows=777, cols=11009, src="f16", fmt="e4m3", block=1, transposed=False),
        # One token through the attention's output projection while serving.
        dict(name="matmul_one_token", op="matmul", m=1, n=4096, k=4096, fmt_a="e4m3", fmt_b="e4m3", block_b=128, out="bf16"),
        # A decoding batch through the up projection: bound by the weights' bytes.
        dict(name="matmul_batch_64", op="matmul", m=64, n=14336, k=4096, fmt_a="e4m3", fmt_b="e4m3", block_b=128, out="bf16"),
        # A ragged prompt through a matrix whose sizes are off every tile.
        dict(name="matmul_ragged", op="matmul", m=777, n=1001, k=2050, fmt_a="e4m3", fmt_b="e4m3", block_b=128, out="f16"),
        # A training step's forward product, 8192 tokens through the up projection: bound by the tensor cores.
        dict(name="matmul_forward", op="matmul", m=8192, n=14336, k=4096, fmt_a="e4m3", fmt_b="e4m3", block_b=128, out="bf16"),
        # The weights' gradient of a key projection over 8192 tokens, to be added up in FP32.
        dict(name="matmul_weight_grad", op="matmul", m=1024, n=4096, k=8192, fmt_a="e5m2", fmt_b="e4m3", block_b=1, out="f32"),
        # One token through a layer of many small experts: latency.
        dict(name="moe_one_token", op="moe", tokens=1, experts=64, top_k=8, hidden=2048, inter=1024, fmt="e4m3", src="bf16"),
        # A decoding batch through the same layer: nearly every expert is read.
        dict(name="moe_batch_64", op="moe", tokens=64, experts=64, top_k=8, hidden=2048, inter=1024, fmt="e4m3", src="bf16"),
        # Few large experts of an 8B-shaped feed-forward layer.
        dict(name="moe_large_experts", op="moe", tokens=16, experts=8, top_k=2, hidden=4096, inter=14336, fmt="e4m3", src="bf16"),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, even over its logarithm, off the round sizes half of the time."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if rng.random() < 0.5 and v >= 64:
        v = v // 64 * 64
    return max(low, min(high, v))


def draw(rng):
    op = rng.choice(["quantize", "matmul", "matmul", "moe"])
    if op == "quantize":
        block = rng.choice([1, 1, 128])
        rows, cols = _spread(rng, 1, 14336), _spread(rng, 64, 14336)
        rows = min(rows, 14336 * 4096 // cols)
        return dict(op=op, rows=rows, cols=cols, src=rng.choice(["f32", "bf16", "f16"]), fmt=rng.choice(["e4m3", "e4m3", "e5m2"]),
                    block=block, transposed=rng.random() < 0.4)
    if op == "matmul":
        n, k = _spread(rng, 64, 14336), _spread(rng, 64, 14336)
        m = min(_spread(rng, 1, 8192), max(1, MOST_FLOPS // (2 * n * k)))
        fmt_a, fmt_b = rng.choice([("e4m3", "e4m3"), ("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
        return dict(op=op, m=m, n=n, k=k, fmt_a=fmt_a, fmt_b=fmt_b, block_b=rng.choice([1, 128]), out=rng.choice(["bf16", "bf16", "f16", "f32"]))
    experts = rng.choice([4, 8, 16, 32, 64, 128])
    hidden = _spread(rng, 512, 4096)
    inter = _spread(rng, 256, max(256, min(14336, 8 * 14336 * 4096 // (experts * hidden))))
    return dict(op=op, tokens=_spread(rng, 1, 64), experts=experts, top_k=rng.choice([1, 2, 4, min(8, experts)]), hidden=hidden, inter=inter,
                fmt=rng.choice(["e4m3", "e4m3", "e5m2"]), src=rng.choice(["bf16", "bf16", "f16"]))


def _ceil(a, b):
    return -(-a // b)


def _blocks(x, block):
    """The matrices x[..., rows, cols], zero padded, as [..., row blocks, rows of a block, column blocks, 128]."""
    rows, cols = x.shape[-2:]
    x = torch.nn.functional.pad(x, (0, -cols % 128, 0, -rows % block))
    return x.reshape(*x.shape[:-2], x.shape[-2] // block, block, x.shape[-1] // 128, 128)


def _quantize(x, fmt, block):
    """(elements, scale bytes) of x[..., rows, cols] in 32 bits."""
    rows, cols = x.shape[-2:]
    xb = _blocks(x.float(), block)
    amax = torch.where(torch.isfinite(xb), xb.abs(), torch.zeros((), device=x.device)).amax(dim=(-3, -1), keepdim=True)
    fraction, exponent = torch.frexp(amax)
    top_fraction, top_exponent = math.frexp(TOP[fmt])
    e = exponent - top_exponent + (fraction > top_fraction).int()
    e = torch.where(amax > 0, e, torch.full_like(e, -127)).clamp(-127, 127)
    q = torch.ldexp(xb, -e).to(FP8[fmt])
    q = q.view(torch.uint8).reshape(*x.shape[:-2], xb.shape[-4] * block, -1)[..., :rows, :cols]
    return q, (e + 127).to(torch.uint8).squeeze(-1).squeeze(-2)


def _values(q, scales, fmt, block):
    """What the elements stand for, in 32 bits."""
    s = torch.ldexp(torch.ones(scales.shape, device=q.device), scales.int() - 127)
    s = s.repeat_interleave(block, dim=-2)[..., : q.shape[-2], :] if block > 1 else s
    s = s.repeat_interleave(128, dim=-1)[..., : q.shape[-1]]
    return q.view(FP8[fmt]).float() * s


def _pitched(q):
    """The matrices with rows of a pitch that is a multiple of 16 bytes."""
    buf = torch.zeros((*q.shape[:-1], _ceil(q.shape[-1], 16) * 16), dtype=torch.uint8, device=q.device)
    out = buf[..., : q.shape[-1]]
    out.copy_(q)
    return out


def _bytes(rows, cols):
    return torch.zeros((rows, _ceil(cols, 16) * 16), dtype=torch.uint8, device=DEVICE)[:, :cols]


def _randn(shape, g):
    return torch.randn(shape, generator=g, device=DEVICE)


def _activations(shape, g):
    """Gaussian values with a few channels (columns) that stand out, as behind a norm."""
    x = _randn(shape, g)
    x[:, torch.randint(shape[1], (max(1, shape[1] // 256),), generator=g, device=DEVICE)] *= 12.0
    return x


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    c = dict(case)
    if own:
        from paper_2508_19263_b200 import binding as zc
    if c["op"] == "quantize":
        rows, cols = c["rows"], c["cols"]
        std = 0.02 if c["block"] == 128 else 1.0 if c["fmt"] == "e4m3" else 1e-4
        x = (_activations((rows, cols), g) if c["block"] == 1 else _randn((rows, cols), g)) * std
        c["x"] = x.to(REAL[c["src"]])
        if own:
            make = lambda r, k: zc.Fp8Matrix(_bytes(r, k), torch.zeros((_ceil(r, c["block"]), _ceil(k, 128)), dtype=torch.uint8, device=DEVICE), FORMAT_CODE[c["fmt"]], c["block"])  # noqa: E731
            c["q"], c["qt"] = make(rows, cols), make(cols, rows) if c["transposed"] else None
        return c
    if c["op"] == "matmul":
        m, n, k = c["m"], c["n"], c["k"]
        a = _activations((m, k), g) if c["fmt_a"] == "e4m3" else _randn((m, k), g) * 1e-4
        b = _randn((n, k), g) * 0.02 if c["block_b"] == 128 else _activations((n, k), g)
        c["a"], c["a_scales"] = _quantize(a, c["fmt_a"], 1)
        c["b"], c["b_scales"] = _quantize(b, c["fmt_b"], c["block_b"])
        c["a"], c["b"] = _pitched(c["a"]), _pitched(c["b"])
        if own:
            c["A"] = zc.Fp8Matrix(c["a"], c["a_scales"], FORMAT_CODE[c["fmt_a"]], 1)
            c["B"] = zc.Fp8Matrix(c["b"], c["b_scales"], FORMAT_CODE[c["fmt_b"]], c["block_b"])
            c["d"] = torch.empty((m, n), dtype=REAL[c["out"]], device=DEVICE)
        return c
    tokens, experts, hidden, inter = c["tokens"], c["experts"], c["hidden"], c["inter"]
    x = torch.zeros((tokens, _ceil(hidden, 8) * 8), dtype=REAL[c["src"]], device=DEVICE)[:, :hidden]
    c["x"] = x.copy_(_activations((tokens, hidden), g) * 0.5)
    r = torch.zeros((experts, _ceil(hidden, 8) * 8), dtype=REAL[c["src"]], device=DEVICE)[:, :hidden]
    c["router"] = r.copy_(_randn((experts, hidden), g) / math.sqrt(hidden))
    c["gate_up"], c["gate_up_scales"] = _quantize(_randn((experts, 2, inter, hidden), g) / math.sqrt(hidden), c["fmt"], 128)
    c["gate_up"] = _pitched(c["gate_up"])
    c["down"], c["down_scales"] = _quantize(_randn((experts, hidden, inter), g) / math.sqrt(inter), c["fmt"], 128)
    c["down"] = _pitched(c["down"])
    if own:
        c["layer"] = zc.Fp8MoeLayer(c["router"], c["gate_up"], c["gate_up_scales"], c["down"], c["down_scales"], c["top_k"], FORMAT_CODE[c["fmt"]])
        c["y"] = torch.empty((tokens, hidden), dtype=REAL[c["src"]], device=DEVICE)
        c["ids"] = torch.empty((tokens, c["top_k"]), dtype=torch.int32, device=DEVICE)
        c["weights"] = torch.empty((tokens, c["top_k"]), dtype=torch.float32, device=DEVICE)
        c["workspace"] = torch.empty(c["layer"].workspace_bytes(tokens), dtype=torch.uint8, device=DEVICE)
    return c


def _run_own(s):
    from paper_2508_19263_b200 import binding as zc
    if s["op"] == "quantize":
        zc.fp8_quantize(s["x"], s["q"], s["qt"])
        return [v for m in (s["q"], s["qt"]) if m is not None for v in (m.elems.view(FP8[s["fmt"]]), m.scales.view(torch.float8_e8m0fnu))]
    if s["op"] == "matmul":
        return zc.fp8_matmul(s["A"], s["B"], s["d"])
    zc.fp8_moe(s["layer"], s["x"], s["y"], s["workspace"], d_ids=s["ids"], d_weights=s["weights"])
    return [s["y"], s["ids"], s["weights"]]


def run(s):
    if own:
        return _run_own(s)
    if s["op"] == "quantize":
        pairs = [_quantize(s["x"], s["fmt"], s["block"])] + ([_quantize(s["x"].t(), s["fmt"], s["block"])] if s["transposed"] else [])
        return [v for q, e in pairs for v in (q.view(FP8[s["fmt"]]), e.view(torch.float8_e8m0fnu))]
    if s["op"] == "matmul":
        a = _values(s["a"], s["a_scales"], s["fmt_a"], 1)
        b = _values(s["b"], s["b_scales"], s["fmt_b"], s["block_b"])
        return torch.matmul(a, b.t()).to(REAL[s["out"]])
    # logits in 64 bits: two experts' may lie next to each other; the sort is stable, so that ties go to the lowest index
    logits = torch.matmul(s["x"].double(), s["router"].double().t())
    order = torch.sort(logits, dim=1, descending=True, stable=True)
    ids, top = order.indices[:, : s["top_k"]], order.values[:, : s["top_k"]]
    weights = torch.exp(top - top[:, :1])
    weights = (weights / weights.sum(dim=1, keepdim=True)).float()
    share = torch.zeros(logits.shape, device=DEVICE).scatter_(1, ids, weights)
    x = s["x"].float()
    gate_up = torch.matmul(x, _values(s["gate_up"], s["gate_up_scales"], s["fmt"], 128).transpose(-1, -2))     # [experts, 2, tokens, inter]
    gate, up = gate_up[:, 0], gate_up[:, 1]
    h = gate / (1.0 + torch.exp(-gate)) * up * share.t().unsqueeze(-1)
    y = torch.matmul(h, _values(s["down"], s["down_scales"], s["fmt"], 128).transpose(-1, -2)).sum(dim=0)
    return [y.to(REAL[s["src"]]), ids.int(), weights]


def work(case):
    c = case
    if c["op"] == "quantize":
        n, times = c["rows"] * c["cols"], 2 if c["transposed"] else 1
        scales = _ceil(c["rows"], c["block"]) * _ceil(c["cols"], 128) + (_ceil(c["cols"], c["block"]) * _ceil(c["rows"], 128) if c["transposed"] else 0)
        return {"bytes": n * (WIDTH[c["src"]] + times) + scales, "flops": 0}
    if c["op"] == "matmul":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": m * k + n * k + (m + _ceil(n, c["block_b"])) * _ceil(k, 128) + m * n * WIDTH[c["out"]], "flops": 2 * m * n * k}
    t, e, top_k, h, i = c["tokens"], c["experts"], c["top_k"], c["hidden"], c["inter"]
    chosen = e * (1.0 - (1.0 - top_k / e) ** t)              # experts that at least one token chooses, on average
    return {"bytes": int(chosen * 3 * h * i * (1 + 1 / 16384) + 2 * e * h + 4 * t * h + 8 * t * top_k), "flops": 2 * t * e * h + 6 * t * top_k * h * i}


# ---- the operators once more, from their definition, in 64 bits -------------------------------------------------------------

def _decoded(fmt):
    """The values of the 256 bytes of a format, from its sign, exponent and mantissa bits."""
    bits, bias = MANTISSA[fmt], BIAS[fmt]
    values = []
    for byte in range(256):
        e, f = (byte & 127) >> bits, byte & ((1 << bits) - 1)
        v = math.ldexp(f, 1 - bias - bits) if e == 0 else math.ldexp(f + (1 << bits), e - bias - bits)
        if fmt == "e4m3" and byte & 127 == 127 or fmt == "e5m2" and e == 31 and f:
            v = math.nan
        elif fmt == "e5m2" and e == 31:
            v = math.inf
        values.append(-v if byte & 128 else v)
    return torch.tensor(values, dtype=torch.float64, device=DEVICE)


def _matrix(elems, scales, fmt, block):
    rows, cols = elems.shape
    row, col = torch.arange(rows, device=DEVICE) // block, torch.arange(cols, device=DEVICE) // 128
    return _decoded(fmt)[elems.long()] * torch.exp2(scales.double() - 127.0)[row][:, col]


def _nearest(x, fmt, block):
    """[elements' values, scales] by the definition: least power of two, then the nearest value, ties to the even one."""
    rows, cols = x.shape
    full = torch.zeros((_ceil(rows, block) * block, _ceil(cols, 128) * 128), dtype=torch.float64, device=DEVICE)
    full[:rows, :cols] = x
    amax = full.abs().reshape(-1, block, full.shape[1] // 128, 128).amax(dim=3).amax(dim=1)
    e = torch.floor(torch.log2(amax.clamp(min=2.0 ** -200) / TOP[fmt])) - 1
    for _ in range(3):
        e = e + (torch.exp2(e) * TOP[fmt] < amax)
    e = torch.where(amax > 0, e.clamp(-127, 127), torch.full_like(e, -127.0))
    scale = torch.exp2(e)
    v = x.double() / scale.repeat_interleave(block, 0)[:rows].repeat_interleave(128, 1)[:, :cols]
    least = 1 - BIAS[fmt]
    # the power of two below |v|: log2 may be off next to one, so it is put right by comparison
    p = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -60)))
    p = p - (torch.exp2(p) > v.abs()).double() + (torch.exp2(p + 1) <= v.abs()).double()
    step = torch.exp2(p.clamp(min=least) - MANTISSA[fmt])
    return [torch.round(v / step) * step, scale]


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "quantize":
        x = s["x"].double()
        return _nearest(x, s["fmt"], s["block"]) + (_nearest(x.t().contiguous(), s["fmt"], s["block"]) if s["transposed"] else [])
    if s["op"] == "matmul":
        return _matrix(s["a"], s["a_scales"], s["fmt_a"], 1) @ _matrix(s["b"], s["b_scales"], s["fmt_b"], s["block_b"]).t()
    x, y = s["x"].double(), torch.zeros(s["x"].shape, dtype=torch.float64, device=DEVICE)
    logits = x @ s["router"].double().t()
    weights = torch.zeros((s["tokens"], s["top_k"]), dtype=torch.float64, device=DEVICE)
    ids = torch.zeros((s["tokens"], s["top_k"]), dtype=torch.int32, device=DEVICE)
    left = logits.clone()
    for j in range(s["top_k"]):
        best = left.max(dim=1, keepdim=True).values
        place = torch.where(left == best, torch.arange(s["experts"], device=DEVICE), s["experts"]).min(dim=1).values
        ids[:, j], weights[:, j] = place.int(), torch.exp(best[:, 0] - logits.max(dim=1).values)
        left[torch.arange(s["tokens"], device=DEVICE), place] = -math.inf
    weights = weights / weights.sum(dim=1, keepdim=True)
    for e in range(s["experts"]):
        token, slot = torch.nonzero(ids == e, as_tuple=True)
        if token.numel():
            gate = x[token] @ _matrix(s["gate_up"][e, 0], s["gate_up_scales"][e, 0], s["fmt"], 128).t()
            up = x[token] @ _matrix(s["gate_up"][e, 1], s["gate_up_scales"][e, 1], s["fmt"], 128).t()
            h = gate * torch.sigmoid(gate) * up
            y.index_add_(0, token, weights[token, slot].unsqueeze(1) * (h @ _matrix(s["down"][e], s["down_scales"][e], s["fmt"], 128).t()))
    return [y, ids, weights]
