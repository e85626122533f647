"""Plain forms in 64 bits of the operators on a quantised key/value cache, and random caches to try them on."""
import math

import torch

FP4, E4M3 = 3, 2
TOP = {FP4: 6.0, E4M3: 448.0}
MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def values(elems, scales, fmt):
    """What elements [..., bytes] with scale bytes [..., blocks] stand for, in FP64."""
    if fmt == E4M3:
        v = elems.view(torch.float8_e4m3fn).double()
    else:
        table = torch.tensor(MAGNITUDES + [-m for m in MAGNITUDES], dtype=torch.float64, device=elems.device)
        v = torch.stack((table[(elems & 15).long()], table[(elems >> 4).long()]), -1).flatten(-2)
    s = torch.exp2(scales.double() - 127)
    s = torch.where(scales == 255, torch.full_like(s, math.nan), s)
    return v * s.repeat_interleave(32, -1)


def quantize(x, fmt):
    """(elements, scale bytes) of finite numbers x[..., dim], by the definition."""
    x = x.double()
    amax = x.reshape(*x.shape[:-1], -1, 32).abs().amax(-1)
    e = torch.full_like(amax, -127.0)
    for _ in range(255):                                       # the least e that will do
        e = torch.where(torch.exp2(e) * TOP[fmt] < amax, e + 1, e)
    y = x / torch.exp2(e).repeat_interleave(32, -1)
    s = (e + 127).to(torch.uint8)
    if fmt == E4M3:                                            # FP64 to E4M3 by way of the nearest multiple of its step
        p = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -9)))
        p = p - (torch.exp2(p) > y.abs()).double() + (torch.exp2(p + 1) <= y.abs()).double()
        step = torch.exp2(p.clamp(min=-6) - 3)
        r = torch.round(y.abs() / step) * step
        return torch.copysign(r, y).float().to(torch.float8_e4m3fn).view(torch.uint8), s
    a = y.abs()
    code = torch.zeros(a.shape, dtype=torch.uint8, device=x.device)
    for i in range(1, 8):
        middle = (MAGNITUDES[i - 1] + MAGNITUDES[i]) / 2
        code += (a > middle) | ((a == middle) & (i % 2 == 0))
    code |= torch.signbit(x).to(torch.uint8) << 3
    return code[..., 0::2] | (code[..., 1::2] << 4), s


class Case:
    """A cache of random bytes with sequences in it; scales between 2^low and 2^high."""

    def __init__(self, zc, fmt, dim, page, kv_heads, lens, new, seed=0, low=-4, high=2, spare=3, more_rows=0, before=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.fmt, self.dim, self.page, self.heads, self.lens_list, self.new = fmt, dim, page, kv_heads, list(lens), list(new)
        used = [-(-n // page) for n in lens]
        pages, places = sum(used) + spare, max(max(used, default=0), 1)
        order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
        table = torch.full((len(lens), places), -1, dtype=torch.int32)            # entries that nobody may read
        at = 0
        for b, n in enumerate(used):
            table[b, :n] = torch.tensor(order[at: at + n], dtype=torch.int32)
            at += n
        self.table, self.spare_pages = table, order[at:]
        self.first_list = [before]
        for n in new:
            self.first_list.append(self.first_list[-1] + n)
        self.rows = self.first_list[-1] + more_rows
        width = dim // 2 if fmt == FP4 else dim

        def elements():
            e = torch.randint(0, 256, (pages, kv_heads, page, width), generator=g, device=device, dtype=torch.uint8)
            return torch.where((e & 127) == 127, e & 0xF0, e) if fmt == E4M3 else e          # no NaN

        def scales():
            return torch.randint(127 + low, 128 + high, (pages, kv_heads, page, dim // 32), generator=g, device=device, dtype=torch.uint8) if low > -127 else \
                torch.randint(0, 255, (pages, kv_heads, page, dim // 32), generator=g, device=device, dtype=torch.uint8)
        self.cache = zc.KvCache(elements(), scales(), elements(), scales(), fmt)
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=device)  # noqa: E731
        self.batch = zc.KvBatch(table.to(device), i32(list(lens)), i32(self.first_list), max(list(new) + [1]))

    def token_slots(self, b):
        """(page, token) of the tokens of sequence b."""
        t = torch.arange(self.lens_list[b])
        return self.table[b, t // self.page].long(), t % self.page

    def tokens(self, b):
        """(K, V) [heads, tokens, dim] of sequence b in FP64."""
        page, token = self.token_slots(b)
        c = self.cache
        take = lambda t: t[page.to(t.device), :, token.to(t.device)].transpose(0, 1)  # noqa: E731
        return values(take(c.k_elems), take(c.k_scales), self.fmt), values(take(c.v_elems), take(c.v_scales), self.fmt)

    def poison(self, causal_window=None):
        """NaN into everything that no token of a sequence occupies, or, with a window, that no row of a causal attention sees."""
        c = self.cache
        mine = torch.zeros(c.k_elems.shape[0], self.page, dtype=torch.bool)
        for b in range(len(self.lens_list)):
            page, token = self.token_slots(b)
            keep = torch.ones(len(page), dtype=torch.bool)
            if causal_window is not None:
                keep = torch.arange(len(page)) > len(page) - self.new[b] - causal_window
            mine[page[keep], token[keep]] = True
        mine = mine.to(c.k_elems.device)
        for e, s in ((c.k_elems, c.k_scales), (c.v_elems, c.v_scales)):
            hide = (~mine)[:, None, :, None]
            e.masked_fill_(hide.expand_as(e), 0x7F)
            s.masked_fill_(hide.expand_as(s), 255)


def attention(case, q, scale, causal=True, window=0, left_out=()):
    """(out, lse, bound) in FP64 of q[rows, q_heads, dim]; rows that are nobody's are NaN.  bound: see `tolerance`.
    left_out: pairs (sequence, place) of pages whose tokens are not seen."""
    rows, q_heads, dim = q.shape
    group = q_heads // case.heads
    out = torch.full(q.shape, math.nan, dtype=torch.float64, device=q.device)
    bound = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.full(q.shape[:2], math.nan, dtype=torch.float64, device=q.device)
    for b, n in enumerate(case.new):
        k, v = case.tokens(b)
        length = case.lens_list[b]
        pos = torch.arange(length - n, length, device=q.device)[:, None]
        t = torch.arange(length, device=q.device)
        seen = (t <= pos) if causal else torch.ones((n, length), dtype=torch.bool, device=q.device)
        if window:
            seen &= t > pos - window
        for s, place in left_out:
            if s == b:
                seen &= (t // case.page != place)
        r = slice(case.first_list[b], case.first_list[b] + n)
        qb = q[r].double().transpose(0, 1).reshape(case.heads, group, n, dim)
        x = torch.einsum("hgnd,htd->hgnt", qb, k) * scale
        x = torch.where(seen, x, torch.full_like(x, -math.inf))
        top = x.amax(-1, keepdim=True) if length else torch.full((*x.shape[:-1], 1), -math.inf, dtype=x.dtype, device=x.device)
        p = torch.exp(x - torch.where(top > -math.inf, top, torch.zeros_like(top)))
        p = torch.where(seen, p, torch.zeros_like(p))
        total = p.sum(-1, keepdim=True)
        p = torch.where(total > 0, p / total, torch.zeros_like(p))
        o = torch.einsum("hgnt,htd->hgnd", p, torch.where(seen.any(0)[:, None], v, torch.zeros_like(v)))
        v_seen, k_seen = (torch.where(seen.any(0)[:, None], z, torch.zeros_like(z)) for z in (v, k))
        terms = torch.einsum("hgnt,htd->hgnd", p, v_seen.abs())
        lost = 2.0 ** -40 * v_seen.abs().sum(1)[:, None, None, :]
        if length:
            top_k, top_v = (z.abs().nan_to_num(0).amax(dim=(1, 2)).reshape(-1, 1, 1, 1) for z in (k_seen, v_seen))
            size = torch.einsum("hgnd,htd->hgnt", qb.abs(), k_seen.abs()).amax(-1, keepdim=True) * abs(scale)
            size = size * 2 * (dim + 8) * 2.0 ** -24 + 2 * abs(scale) * qb.abs().sum(-1, keepdim=True) * top_k * 2.0 ** -31
            lost = lost + 2.0 ** -31 * top_v
        else:
            size = torch.zeros_like(top)
        back = lambda z: z.transpose(1, 2).transpose(0, 1).reshape(n, q_heads, z.shape[-1]) if n else z.reshape(0, q_heads, z.shape[-1])  # noqa: E731
        out[r], lse[r] = back(o), back(top + torch.log(total))[..., 0]
        bound[r] = back(terms * (2.0 ** -12 + max(4096, length) * 2.0 ** -24 + size) + lost)
    return out, lse, bound


def tolerance(want, bound, dtype):
    """How far a result may be off: half a step of its type, and `bound`.  With p the weights, each is off by 2^-12 where it is rounded to FP16, and their
    sums over n terms in FP32 by n 2^-24 (n taken as 4096 at least: 2^-12).  Weights go into FP16 times 2^15 over the row's largest: what is below its least subnormal, 2^-24, is off by
    half of that, 2^-40 of the largest weight, for each value.  A logit of `dim` products summed in FP32 is off by (dim + 8) 2^-24 of its terms' magnitudes, which moves a weight, and the sum
    that it is divided by, by as much.  Keys and values go into FP16 over a power of two so that the largest of a head is at least 2^(15 - 9): E4M3 spans
    2^-9 .. 448 < 2^9 times its scale; below FP16's least subnormal they are off by half of it, 2^-25 / 2^6 = 2^-31 of the largest.
    The least subnormals of FP16 results are 2^-24, and FP32's least normal number, 2^-126, bounds what is lost of BF16 ones."""
    return torch.finfo(dtype).eps / 2 * want.abs() * (1 + 2.0 ** -9) + bound + (2.0 ** -25 if dtype == torch.float16 else 2.0 ** -126)
