"""Attention over a quantised key/value cache against the formula in 64 bits."""
import math

import pytest
import torch

import kv_reference as ref
from paper_2508_19263_b200 import binding as zc

pytestmark = pytest.mark.gpu
FP4, E4M3 = zc.FMT_FP4_E2M1, zc.FMT_FP8_E4M3
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def clean():
    zc.kv_status()
    yield
    assert zc.kv_status() == zc.OK


def queries(case, group, dtype, seed=11, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((case.rows, case.heads * group, case.dim), generator=g, device="cuda") * size).to(dtype)


def workspace(case, q_heads):
    return torch.randint(0, 256, (zc.kv_attention_workspace_bytes(case.cache, case.batch, q_heads),), dtype=torch.uint8, device="cuda")


def check(case, q, scale=None, causal=True, window=0, left_out=(), out=None):
    real = case.dim ** -0.5 if scale is None else scale
    out = torch.full_like(q, 7.0) if out is None else out
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    zc.kv_attention(case.cache, case.batch, q, out, workspace(case, q.shape[1]), scale=scale, causal=causal, window=window, d_lse=lse)
    want, want_lse, bound = ref.attention(case, q, real, causal, window, left_out)
    mine = torch.zeros(case.rows, dtype=torch.bool, device="cuda")
    mine[case.first_list[0]: case.first_list[-1]] = True
    assert bool((out[~mine] == 7.0).all()) and bool((lse[~mine] == 7.0).all()), "rows that are nobody's"
    off = (out.double() - want).abs() - ref.tolerance(want, bound, q.dtype)
    assert bool((off[mine] <= 0).all()), f"off by {off[mine].max().item():.3g} too much"
    none = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(lse) & mine[:, None], none) and bool((out[none] == 0).all()) and bool((lse[none] == -math.inf).all())
    seen = mine[:, None] & ~none
    # a logit is off by (dim + 8) 2^-24 of its terms' magnitudes (the bound's second part), sum and logarithm by 2^-20
    lse_off = (lse.double() - want_lse).abs()
    room = 2.0 ** -20 * (1 + want_lse.abs()) + (case.dim + 8) * 2.0 ** -24 * logit_size(case, q, real)
    assert bool((lse_off[seen] <= room[seen]).all()), f"lse off by {(lse_off - room)[seen].max().item():.3g} too much"
    return out, lse


def logit_size(case, q, scale):
    size = torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    for b, n in enumerate(case.new):
        k = torch.nan_to_num(case.tokens(b)[0]).abs()
        if k.shape[1] == 0 or n == 0:
            continue
        r = slice(case.first_list[b], case.first_list[b] + n)
        top = k.amax(1).repeat_interleave(q.shape[1] // case.heads, 0)
        size[r] = (q[r].double().abs() * top).sum(-1) * abs(scale)
    return size


@pytest.mark.parametrize("fmt", [FP4, E4M3])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim,page,heads,group,lens", [
    (128, 16, 8, 4, [1]), (64, 16, 1, 1, [1, 2, 15, 16, 17]), (128, 16, 2, 8, [31, 32, 33, 63, 64, 65, 0, 100]), (128, 64, 3, 7, [1000, 129, 500]),
    (64, 32, 5, 3, [700, 1, 257, 511]), (128, 128, 1, 16, [4000]), (64, 256, 2, 12, [777, 300]), (128, 32, 2, 40, [200, 90]), (64, 16, 1, 256, [50])])
def test_single_tokens(fmt, dtype, dim, page, heads, group, lens):
    case = ref.Case(zc, fmt, dim, page, heads, lens, [1] * len(lens), more_rows=2, before=1)
    case.poison()
    check(case, queries(case, group, dtype))


@pytest.mark.parametrize("fmt", [FP4, E4M3])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim,page,heads,group,lens,new", [
    (128, 16, 2, 4, [40, 3, 100], [2, 3, 4]), (64, 16, 1, 1, [16, 17, 18], [16, 1, 18]), (128, 64, 2, 4, [300, 64, 0, 129], [300, 5, 0, 1]), (64, 32, 3, 5, [777, 100], [333, 100]),
    (128, 32, 1, 8, [1500], [257]), (128, 16, 4, 1, [129, 128, 127], [129, 128, 127]), (64, 128, 1, 16, [260], [130]), (128, 16, 1, 3, [2048], [43])])
@pytest.mark.parametrize("causal", [True, False])
def test_several_rows(fmt, dtype, dim, page, heads, group, lens, new, causal):
    case = ref.Case(zc, fmt, dim, page, heads, lens, new, more_rows=1, before=3)
    case.poison()
    check(case, queries(case, group, dtype), causal=causal)


@pytest.mark.parametrize("fmt,dtype", [(FP4, BF16), (E4M3, F16)])
@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 100, 5000])
@pytest.mark.parametrize("new", [[1, 1, 1], [3, 2, 1], [200, 64, 33]])
def test_window(fmt, dtype, window, new):
    case = ref.Case(zc, fmt, 64, 16, 2, [500, 64, 33], new)
    case.poison(causal_window=window)
    check(case, queries(case, 4, dtype), window=window)


@pytest.mark.parametrize("new", [[3, 5, 2, 1], [200, 40, 64, 1]])
@pytest.mark.parametrize("causal", [True, False])
def test_rows_that_see_nothing(new, causal):
    # fewer tokens than rows: the first rows have negative positions; sequences without tokens
    case = ref.Case(zc, FP4, 128, 16, 2, [1, 0, 2, 0], new, more_rows=1)
    check(case, queries(case, 4, BF16), causal=causal)


@pytest.mark.parametrize("fmt", [FP4, E4M3])
@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("scale,size", [(-0.1, 1.0), (0.0, 1.0), (3.0, 1.0), (2.0 ** -30, 2.0 ** 20), (0.5, 2.0 ** -120)])
def test_scales_and_sizes(fmt, new, scale, size):
    case = ref.Case(zc, fmt, 64, 16, 2, [300], [new])
    check(case, queries(case, 4, BF16, size=size), scale=scale)


@pytest.mark.parametrize("fmt", [FP4, E4M3])
@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("low,high", [(-14, 2), (-60, -50), (0, 9), (40, 45), (-4, -4)])
def test_wide_scales(fmt, new, low, high):
    # scale bytes far apart, far from 1; the queries keep the logits within reach
    case = ref.Case(zc, fmt, 128, 32, 2, [333, 65], [new, 1], low=low, high=high)
    case.cache.v_scales.copy_(case.cache.v_scales.flip(0))
    check(case, queries(case, 4, BF16, size=2.0 ** -high / 8))


@pytest.mark.parametrize("new", [1, 70])
def test_sharp_softmax(new):
    # logits of several hundreds: all but a few weights vanish
    case = ref.Case(zc, FP4, 128, 16, 1, [900], [new])
    check(case, queries(case, 8, F16), scale=8.0)


@pytest.mark.parametrize("new", [[1, 1], [66, 2]])
def test_strides(new):
    case = ref.Case(zc, FP4, 128, 16, 2, [200, 70], new)
    rows, heads = case.rows, 8
    plain = queries(case, 4, BF16)
    for shape, order in (((heads, rows, 128), (1, 0, 2)), ((rows, 3, heads, 128), None), ((rows, heads, 129), "odd")):
        room = torch.full(shape, 7.0, dtype=BF16, device="cuda")
        view = (lambda t: t.permute(order)) if isinstance(order, tuple) else (lambda t: t[:, 1]) if order is None else (lambda t: t[..., 1:])
        q = view(room.clone())
        q.copy_(plain)
        out = view(room)
        check(case, q, out=out)
        keep = torch.full(shape, 7.0, dtype=BF16, device="cuda")
        view(keep).copy_(out)
        assert torch.equal(room, keep)


@pytest.mark.parametrize("new", [1, 80])
def test_nan_is_seen_where_it_counts_and_nowhere_else(new):
    case = ref.Case(zc, E4M3, 64, 16, 2, [100, 100], [new, new])
    q = queries(case, 2, BF16)
    ws = workspace(case, 4)
    want = zc.kv_attention(case.cache, case.batch, q, torch.empty_like(q), ws).clone()
    page = case.table[1, 1].item()
    case.cache.k_scales[page, 1, 3, 0] = 255                    # a key of the second sequence's second head, position 19
    got = zc.kv_attention(case.cache, case.batch, q, torch.empty_like(q), ws)
    pos = torch.arange(100 - new, 100)
    hit = torch.zeros((2 * new, 4), dtype=torch.bool)
    hit[new:, 2:] = (pos >= 19)[:, None]
    assert torch.equal(torch.isnan(got).all(-1).cpu(), hit)
    assert torch.equal(got[~hit.cuda()], want[~hit.cuda()])
    q[0, 0, 5] = math.nan                                        # one query's
    got = zc.kv_attention(case.cache, case.batch, q, torch.empty_like(q), ws)
    hit[0, 0] = True
    assert torch.equal(torch.isnan(got).any(-1).cpu(), hit)
    assert torch.equal(got[~hit.cuda()], want[~hit.cuda()])


@pytest.mark.parametrize("new", [1, 80])
def test_bad_pages_are_left_out(new):
    case = ref.Case(zc, FP4, 64, 16, 2, [130, 90], [new, 1])
    q = queries(case, 4, BF16)
    case.batch.page_table[0, 2], case.batch.page_table[1, 0] = case.cache.n_pages, -2
    check(case, q, left_out=((0, 2), (1, 0)))
    assert zc.kv_status() == zc.E_CORRUPT and zc.kv_status() == zc.OK


def test_bad_lengths_and_first_rows_are_not_followed():
    case = ref.Case(zc, FP4, 64, 16, 2, [40, 20], [5, 70])
    q = queries(case, 4, BF16)
    case.batch.page_table.clamp_(min=0)
    for lens, first in (([-3, 1 << 30], [0, 5, 75]), ([40, 20], [0, 1 << 30, 75]), ([40, 20], [-(1 << 31), 5, (1 << 31) - 1]), ([40, 20], [60, 30, 10]), ([40, 20], [1 << 30, 5, 75])):
        case.batch.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        case.batch.first.copy_(torch.tensor(first, dtype=torch.int32))
        zc.kv_attention(case.cache, case.batch, q, torch.empty_like(q), workspace(case, 8))
        k = torch.empty((case.rows, 2, 64), dtype=BF16, device="cuda")
        zc.kv_read(case.cache, case.batch, k, None)
        zc.kv_status()


@pytest.mark.parametrize("new,lens", [([1] * 5, [3000, 10, 700, 0, 4096]), ([130, 1, 7], [1000, 3000, 700])])
def test_the_same_every_time(new, lens):
    case = ref.Case(zc, FP4, 128, 16, 4, lens, new)
    q = queries(case, 4, BF16)
    outs = [zc.kv_attention(case.cache, case.batch, q, torch.empty_like(q), workspace(case, 16)) for _ in range(4)]
    assert all(torch.equal(o, outs[0]) for o in outs)


@pytest.mark.parametrize("new", [1, 90])
def test_captured_calls_follow_lengths_and_streams(new):
    # one graph, other lengths at every replay; next to it an eager call on another stream with a workspace of its own
    case = ref.Case(zc, FP4, 128, 16, 2, [700, 333], [new, new])
    q = queries(case, 4, BF16)
    out, ws = torch.empty_like(q), workspace(case, 8)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        zc.kv_attention(case.cache, case.batch, q, out, ws)
    other, ws2 = torch.empty_like(q), workspace(case, 8)
    for lens in ([700, 333], [650, 90], [90, 100], [0, 1]):
        case.batch.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        case.lens_list = lens
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            graph.replay()
        zc.kv_attention(case.cache, case.batch, q, other, ws2)
        torch.cuda.synchronize()
        assert torch.equal(out, other)
        want, _, bound = ref.attention(case, q, 128 ** -0.5)
        assert bool(((out.double() - want).abs() <= ref.tolerance(want, bound, BF16)).all())


@pytest.mark.parametrize("max_new", [0, 1, 8, 64, 100000])
def test_max_new_changes_no_result_beyond_rounding(max_new):
    case = ref.Case(zc, FP4, 64, 16, 2, [300, 90, 40], [100, 1, 9])
    case.batch = zc.KvBatch(case.batch.page_table, case.batch.lens, case.batch.first, max_new)
    check(case, queries(case, 4, BF16))


def test_a_run_of_them():
    # prompts, then single tokens: written, attended over, and the cache's pages through the codec and back in between
    heads, group, dim, page = 2, 4, 64, 16
    case = ref.Case(zc, FP4, dim, page, heads, [70, 33], [70, 33], spare=6)
    table = torch.full((2, 8), -1, dtype=torch.int32)
    table[:, : case.table.shape[1]] = case.table
    spare = list(case.spare_pages)
    for b, n in enumerate(case.lens_list):                       # room for the tokens to come
        for place in range(-(-n // page), -(-(n + 20) // page)):
            table[b, place] = spare.pop()
    case.table = table
    lens, new = [70, 33], [70, 33]
    for step in range(20):
        g = torch.Generator(device="cuda").manual_seed(step)
        case.lens_list, case.new, case.first_list = lens, new, [0, new[0], new[0] + new[1]]
        case.rows = case.first_list[-1]
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        case.batch = zc.KvBatch(table.cuda(), i32(lens), i32(case.first_list), max(new))
        qkv = torch.randn((case.rows, heads * (group + 2), dim), generator=g, device="cuda").to(BF16)
        q, k, v = qkv[:, : heads * group], qkv[:, heads * group: heads * (group + 1)], qkv[:, heads * (group + 1):]
        zc.kv_append(case.cache, case.batch, k, v)
        for x, side in ((k, 0), (v, 1)):
            for b in range(2):
                rows = slice(case.first_list[b], case.first_list[b + 1])
                want = ref.values(*ref.quantize(x[rows], FP4), FP4).transpose(0, 1)
                assert torch.equal(case.tokens(b)[side][:, -new[b]:], want)
        out, _ = check(case, q)
        if step % 7 == 0:
            c, kept = case.cache, []
            for t, fmt in ((c.k_elems, zc.FMT_FP4_E2M1), (c.v_elems, zc.FMT_FP4_E2M1), (c.k_scales, zc.FMT_SCALE_U8), (c.v_scales, zc.FMT_SCALE_U8)):
                data = t.reshape(-1)
                p = zc.plan(fmt, data.numel() * (2 if fmt == zc.FMT_FP4_E2M1 else 1), 4096)
                cb = zc.build_codebook(p, zc.histogram(p, data).cpu().numpy(), zc.POLICY_AUTO)
                packed, ws = torch.empty(p.max_compressed_bytes, dtype=torch.uint8, device="cuda"), torch.empty(p.workspace_bytes, dtype=torch.uint8, device="cuda")
                size = zc.compress(p, cb, data, packed, ws)
                kept.append((t, p, packed, size, ws))
            for t, *_ in kept:
                t.fill_(0xEE)
            for t, p, packed, size, ws in kept:
                zc.decompress(p, packed, size, t.reshape(-1), ws)
                assert zc.device_status(p, ws) == zc.OK
            again = zc.kv_attention(case.cache, case.batch, q, torch.empty_like(out), workspace(case, heads * group))
            assert torch.equal(again, out)
        lens, new = [n + 1 for n in lens], [1, 1]
