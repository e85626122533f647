"""Attention over a quantised key/value cache at the ends of FP32's range, and what it does not touch."""
import math

import pytest
import torch

import kv_reference as ref
from paper_2508_19263_b200 import binding as zc
from test_gpu_kv_attention import BF16, E4M3, F16, FP4, check, clean, queries, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


def big_logits(fmt, new, lens, group, least, loud, dtype=BF16, seed=3):
    """A case whose keys are all the same but for one token of each sequence, `loud` times as large, and queries along the key, of both signs, twice as large with
    every pair of heads: logits are exact in FP32 (whole multiples of a quarter below 2^24, over a power of two) up to the scale, from 2^least on, and far apart where they differ."""
    case = ref.Case(zc, fmt, 128, 16, 2, lens, new, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    grid = torch.tensor(ref.MAGNITUDES, device="cuda")
    key = grid[torch.randint(0, 8, (2, 128), generator=g, device="cuda")] * torch.randint(0, 2, (2, 128), generator=g, device="cuda").mul(2).sub(1)
    every = zc.KvBatch(case.batch.page_table.clamp(min=0), case.batch.lens, torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32, device="cuda"), max(lens))
    k = key.expand(sum(lens), 2, 128).clone()
    at = 0
    for n in lens:
        if loud != 1 and n > 5:
            k[at + 5] *= loud                                     # all rows see it
        at += n
    v = torch.randn(k.shape, generator=g, device="cuda") * 0.25 + 1.0
    zc.kv_append(case.cache, every, k.to(BF16), v.to(BF16))
    heads = 2 * group
    power = torch.exp2(torch.arange(heads, device="cuda") // 2 % max(1, group // 2)).float()
    sign = 1.0 - 2.0 * (torch.arange(heads, device="cuda") % 2)
    q = (key.repeat_interleave(group, 0) * (power * sign)[:, None]).expand(case.rows, heads, 128).to(dtype).contiguous()
    # the least of the logits is scale * |key|^2
    scale = 1.1 * 2.0 ** least / (key * key).sum(-1).min().item()
    return case, q, scale


def check_exact_logits(case, q, scale):
    """Weights are 0 or all the same: what is off is half a step of the result, FP32 sums over the tokens (n 2^-24, n taken as 4096 at least) and the weights' rounding."""
    out, lse = torch.full_like(q, 7.0), torch.zeros(q.shape[:2], device="cuda")
    zc.kv_attention(case.cache, case.batch, q, out, workspace(case, q.shape[1]), scale=scale, d_lse=lse)
    scale = torch.tensor(scale, dtype=torch.float32).double().item()
    want, want_lse, _ = ref.attention(case, q, scale)
    top = torch.cat([case.tokens(b)[1].abs().amax(dim=(1, 2)).max().expand(n) for b, n in enumerate(case.new)])[:, None, None]
    room = torch.finfo(q.dtype).eps / 2 * want.abs() * (1 + 2.0 ** -9) + top * (2.0 ** -12 + 2.0 ** -12)
    off = (out.double() - want).abs() - room
    assert bool((off <= 0).all()), f"{(~(off <= 0)).sum().item()} of {off.numel()} results are off, {torch.isnan(out).sum().item()} are NaN"
    # scale in FP32 and times log2(e), the product, and back: six roundings of 2^-24 and log2(e) itself
    assert bool(((lse.double() - want_lse).abs() <= 2.0 ** -21 * want_lse.abs() + 2.0 ** -19).all())


@pytest.mark.parametrize("fmt", [FP4, E4M3])
@pytest.mark.parametrize("new,lens", [([1, 1], [40, 700]), ([3, 1], [300, 20]), ([70, 33], [300, 129]), ([1], [9000])])
@pytest.mark.parametrize("least,group", [(8, 4), (12, 16), (20, 16), (24, 2), (25, 16), (30, 8), (33, 16), (60, 32), (100, 16)])
@pytest.mark.parametrize("loud", [1, 2])
def test_large_logits(fmt, new, lens, least, group, loud):
    case, q, scale = big_logits(fmt, new, lens, group, least, loud)
    check_exact_logits(case, q, scale)


@pytest.mark.parametrize("new", [1, 3, 70])
@pytest.mark.parametrize("fmt,low,high", [(FP4, 60, 64), (FP4, 100, 105), (FP4, 110, 113), (FP4, 114, 118), (FP4, 116, 120), (FP4, 119, 124), (E4M3, 95, 100), (E4M3, 100, 105), (E4M3, 110, 115), (E4M3, 117, 119),
                                          (FP4, -115, -110), (FP4, -120, -114), (E4M3, -110, -100), (E4M3, -120, -112), (E4M3, 90, 112), (FP4, 80, 118), (FP4, -40, 100), (FP4, -126, 110)])
def test_key_scales_over_all_of_their_range(new, fmt, low, high):
    # queries at the keys' inverse: ordinary logits, whichever kernel has them
    case = ref.Case(zc, fmt, 128, 32, 2, [333, 65], [new, 1], low=low, high=high)
    case.cache.v_scales.random_(124, 129, generator=torch.Generator(device="cuda").manual_seed(1))
    size = 2.0 ** (-high - 3) if fmt == FP4 else 2.0 ** (-high - 6)
    check(case, queries(case, 4, BF16, size=size))


@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("fmt,shift", [(FP4, 112), (FP4, 116), (FP4, 120), (E4M3, 105), (E4M3, 112), (E4M3, 115)])
def test_tiny_queries_are_not_rounded_up(new, fmt, shift):
    # the same logits by keys 2^shift times as large and queries 2^-shift times: the same results
    case = ref.Case(zc, fmt, 128, 16, 2, [500], [new], low=-4, high=-1)
    q = torch.sign(queries(case, 4, BF16)) * 2.0 ** -5
    ws = workspace(case, 8)
    want = zc.kv_attention(case.cache, case.batch, q, torch.empty_like(q), ws)
    case.cache.k_scales.add_(shift)
    got = zc.kv_attention(case.cache, case.batch, q * 2.0 ** -shift, torch.empty_like(q), ws)
    assert torch.equal(got, want)


@pytest.mark.parametrize("lens,new", [([333, 65], [1, 1]), ([333, 65], [70, 1]), ([20000], [1]), ([5000], [64])])
@pytest.mark.parametrize("fmt,low,high", [(FP4, 60, 64), (FP4, 118, 124), (FP4, 123, 124), (E4M3, 110, 118), (E4M3, 117, 118)])
def test_value_scales_over_all_of_their_range(lens, new, fmt, low, high):
    # sums of values that are far beyond FP32, means that are not
    case = ref.Case(zc, fmt, 128, 16, 2, lens, new, low=low, high=high)
    case.cache.k_scales.random_(120, 124, generator=torch.Generator(device="cuda").manual_seed(1))
    case.cache.v_elems.bitwise_and_(0x77 if fmt == FP4 else 0x7F)                    # of one sign
    out, _ = check(case, queries(case, 4, BF16))
    assert bool(torch.isfinite(out).all())


def test_a_half_that_waits_for_its_rows_does_not_give_up():
    # 40 columns a sequence leave the second half of a tile of 256 without rows, for all of a block's work but the last sequence's: hundreds of steps, with a limit that is
    # many times a step's (16 polls do for the sequences of 40 alone)
    seqs, tokens, page = 1500, 16384, 256
    cache = zc.kv_empty(tokens // page, 1, page, 64, FP4)
    g = torch.Generator(device="cuda").manual_seed(1)
    for t in (cache.k_elems, cache.v_elems):
        t.random_(0, 256, generator=g)
    for t in (cache.k_scales, cache.v_scales):
        t.fill_(125)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.arange(tokens // page, dtype=torch.int32, device="cuda").expand(seqs, -1).contiguous()        # they share their pages
    try:
        for last in (40, 256):
            first = [40 * b for b in range(seqs)] + [40 * (seqs - 1) + last]
            batch = zc.KvBatch(table, i32([tokens] * seqs), i32(first), 256)
            q = torch.randn((first[-1], 1, 64), generator=g, device="cuda").to(BF16)
            ws = torch.empty(zc.kv_attention_workspace_bytes(cache, batch, 1), dtype=torch.uint8, device="cuda")
            zc.test_set_wait_limit(0)
            want = zc.kv_attention(cache, batch, q, torch.empty_like(q), ws)
            assert zc.kv_status() == zc.OK
            zc.test_set_wait_limit(64)
            got = zc.kv_attention(cache, batch, q, torch.empty_like(q), ws)
            assert zc.kv_status() == zc.OK
            assert torch.equal(got, want)
    finally:
        zc.test_set_wait_limit(0)


def test_rows_that_are_nobodys_are_not_read():
    # a tensor with room for 262144 tokens: where the batch has one of them, writing takes a small part of the time that writing all of them takes (reading them alone would take most of it)
    rows, heads, page = 1 << 18, 8, 256
    cache = zc.kv_empty(rows // page, heads, page, 128, FP4)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.arange(rows // page, dtype=torch.int32, device="cuda").reshape(1, -1)
    k = torch.ones((rows, heads, 128), device="cuda")
    times = []
    for first in ([0, rows], [5, 6], [rows - 1, rows]):
        batch = zc.KvBatch(table, i32([rows]), i32(first), 1)
        zc.kv_append(cache, batch, k, k)
        events = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        events[0].record()
        for _ in range(10):
            zc.kv_append(cache, batch, k, k)
        events[1].record()
        torch.cuda.synchronize()
        times.append(events[0].elapsed_time(events[1]))
    assert max(times[1:]) * 4 < times[0], times


@pytest.mark.parametrize("dim,columns", [(128, 48), (128, 49), (64, 64), (64, 65)])
def test_both_sides_of_the_choice_of_kernels(dim, columns):
    # the most columns of the kernel of few rows, the least of that of many, alone and with sequences of the other kind beside them; the pages beyond 4 GB
    pages, heads, page = (1 << 32) // (8 * 64 * dim // 2) + 40, 8, 64
    cache = zc.KvCache(*[torch.zeros((pages, heads, page, w), dtype=torch.uint8, device="cuda") for w in (dim // 2, dim // 32, dim // 2, dim // 32)], FP4)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    lens = [300, 200, 77]
    table = torch.full((3, 5), -1, dtype=torch.int32)
    for b, n in enumerate(lens):
        used = -(-n // page)
        table[b, :used] = pages - 1 - 10 * b - torch.arange(used, dtype=torch.int32)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((sum(lens), heads, dim), generator=g, device="cuda").to(BF16) for _ in range(2))
    zc.kv_append(cache, zc.KvBatch(table.cuda(), i32(lens), i32([0, 300, 500, 577]), 300), k, v)
    kv = [ref.values(*ref.quantize(t, FP4), FP4) for t in (k, v)]
    for new in ([columns, columns, columns], [columns, 1, 70], [1, columns, 3]):
        first = [0, new[0], new[0] + new[1], sum(new)]
        batch = zc.KvBatch(table.cuda(), i32(lens), i32(first), columns)
        q = torch.randn((sum(new), heads, dim), generator=g, device="cuda").to(BF16)
        out = torch.empty_like(q)
        zc.kv_attention(cache, batch, q, out, torch.empty(zc.kv_attention_workspace_bytes(cache, batch, heads), dtype=torch.uint8, device="cuda"))
        at = 0
        for b, n in enumerate(new):
            kb, vb = (t[at: at + lens[b]] for t in kv)
            at += lens[b]
            x = torch.einsum("rhd,thd->hrt", q[first[b]: first[b + 1]].double(), kb) * dim ** -0.5
            x = x.masked_fill(torch.arange(lens[b], device="cuda") > torch.arange(lens[b] - n, lens[b], device="cuda")[:, None], -math.inf)
            want = torch.einsum("hrt,thd->rhd", torch.softmax(x, -1), vb)
            # half a step of BF16; 2^-12 for the weights, as much for their sums, 2^-12 for logits of a few units in FP32
            assert bool(((out[first[b]: first[b + 1]].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -10 * vb.abs().amax(0)).all())


@pytest.mark.parametrize("columns,steps,width,max_new", [(8 * (1 << 18), 1776 << 14, 64, 1), (256 * (1 << 16), 148 << 16, 128, 1 << 24)])
def test_calls_of_hours_are_not_begun(columns, steps, width, max_new):
    # one page of zeros is all of a sequence of some 10^9 tokens: 2^32 steps for each warp of 148 blocks of 12 (few rows), for each of 148 blocks (many).  Counted in 32 bits that
    # would be none at all, and for other numbers of blocks it could be hours, so it is for this one alone
    if torch.cuda.get_device_properties(0).multi_processor_count != 148:
        pytest.skip("the sizes are those of 148 multiprocessors")
    cache = zc.kv_empty(1, 1, 256, 64, FP4)
    for t in (cache.k_elems, cache.k_scales, cache.v_elems, cache.v_scales):
        t.zero_()
    table = torch.zeros((1, -(-steps * width // 256)), dtype=torch.int32, device="cuda")
    batch = zc.KvBatch(table, torch.tensor([steps * width], dtype=torch.int32, device="cuda"), torch.tensor([0, columns], dtype=torch.int32, device="cuda"), max_new)
    q = torch.zeros((columns, 1, 64), dtype=BF16, device="cuda")
    out = torch.full_like(q, 7.0)
    zc.kv_attention(cache, batch, q, out, torch.empty(zc.kv_attention_workspace_bytes(cache, batch, 1), dtype=torch.uint8, device="cuda"), causal=False)
    assert zc.kv_status() == zc.E_DEVICE_TIMEOUT
    # the next call is not disturbed
    small = zc.KvBatch(table, torch.tensor([100], dtype=torch.int32, device="cuda"), torch.tensor([0, 3], dtype=torch.int32, device="cuda"), max_new)
    zc.kv_attention(cache, small, q[:3], out[:3], torch.empty(zc.kv_attention_workspace_bytes(cache, small, 1), dtype=torch.uint8, device="cuda"))
    assert zc.kv_status() == zc.OK and bool((out[:3] == 0).all())


@pytest.mark.parametrize("fmt", [FP4, E4M3])
@pytest.mark.parametrize("new,lens", [([1, 1], [40, 700]), ([3, 1], [300, 20]), ([70, 33], [300, 129]), ([1], [9000])])
def test_a_weight_of_one_is_exact(fmt, new, lens):
    # where one token has all of the weight the result is its value, to the bit: in FP16, which has the cache's elements exactly, half a step is 2^-12
    case, q, scale = big_logits(fmt, new, lens, 4, 8, 2, F16)
    out = zc.kv_attention(case.cache, case.batch, q, torch.empty_like(q), workspace(case, 8), scale=scale)
    for b, n in enumerate(new):
        v = case.tokens(b)[1][:, 5]                                # [heads of the cache][dim]; the queries of even heads point to it
        rows = slice(case.first_list[b], case.first_list[b] + n)
        assert torch.equal(out[rows, 0::2].double(), v.repeat_interleave(2, 0).expand(n, 4, 128))
