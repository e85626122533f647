"""Writing a quantised key/value cache and reading it back: bit for bit against the definition in 64 bits."""
import math

import pytest
import torch

import kv_reference as ref
from paper_2508_19263_b200 import binding as zc

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
FORMATS = [zc.FMT_FP4_E2M1, zc.FMT_FP8_E4M3]


@pytest.fixture(autouse=True)
def clean():
    zc.kv_status()
    yield
    assert zc.kv_status() == zc.OK


def numbers(shape, dtype, seed, spread=6):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(shape, generator=g, device="cuda") * torch.exp2(torch.randint(-spread, spread + 1, shape[:-1] + (1,), generator=g, device="cuda").float())
    return x.to(dtype)


def expected(case, before, x, name):
    """The cache's (elements, scales) once the rows of x are in it."""
    elems, scales = (t.clone() for t in before)
    e, s = ref.quantize(x, case.fmt)
    for b, n in enumerate(case.new):
        page, token = case.token_slots(b)
        keep = min(n, case.lens_list[b])
        r = case.first_list[b] + n - keep
        page, token = page[len(page) - keep:].cuda(), token[len(token) - keep:].cuda()
        elems[page, :, token], scales[page, :, token] = e[r: r + keep], s[r: r + keep]
    return elems, scales


def parts(c):
    return {"k": (c.k_elems, c.k_scales), "v": (c.v_elems, c.v_scales)}


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim,page,heads,lens,new", [
    (64, 16, 1, [1], [1]), (128, 16, 8, [17, 16, 1, 0, 40], [1, 1, 1, 0, 1]), (128, 32, 3, [100, 33, 0, 64], [100, 2, 0, 31]),
    (64, 256, 5, [513, 300], [513, 44]), (128, 64, 2, [5, 3], [9, 3]),               # more rows than tokens: the first four have no place
    (64, 128, 4, [7000], [6999])])
def test_append_and_read(fmt, dtype, dim, page, heads, lens, new):
    case = ref.Case(zc, fmt, dim, page, heads, lens, new, more_rows=3, before=2)
    k, v = numbers((case.rows, heads, dim), dtype, 1), numbers((case.rows, heads, dim), dtype, 2)
    before = {n: [t.clone() for t in p] for n, p in parts(case.cache).items()}
    zc.kv_append(case.cache, case.batch, k, v)
    for name, x in (("k", k), ("v", v)):
        for got, want in zip(parts(case.cache)[name], expected(case, before[name], x, name)):
            assert torch.equal(got, want), name
    out = [torch.full_like(k, 7.0), torch.full_like(k, 7.0)]
    zc.kv_read(case.cache, case.batch, *out)
    for side, got in enumerate(out):
        want = torch.full_like(got, 7.0)
        for b, n in enumerate(new):
            t = case.tokens(b)[side].transpose(0, 1)[max(0, lens[b] - n):]
            r = case.first_list[b]
            want[r: r + n] = torch.cat([torch.zeros((n - len(t), heads, dim), dtype=torch.float64, device="cuda"), t]).to(dtype)
        assert torch.equal(got, want)
    again = torch.full_like(k, 7.0)
    zc.kv_read(case.cache, case.batch, None, again)
    assert torch.equal(again, out[1])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
def test_every_tie_and_every_size(fmt, dtype):
    # a block's largest element from the least to the greatest power of two, with all middles between neighbouring values of the format below it
    steps = torch.tensor([0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, .2499, .2501, 5.01, 4.99, .01, -.25, -.75, -1.25, -2.5, -3.5, -5, -0.0, -.1, .1, 1e-3, 0, 0])
    if fmt == zc.FMT_FP8_E4M3:
        steps = steps * 74.0 + torch.arange(32) * 2.0 ** -10
    exps = list(range(-140, 121)) if dtype != torch.float16 else list(range(-24, 13))
    rows = -(-len(exps) // 4)
    x = torch.zeros((rows, 1, 128))
    for i, e in enumerate(exps):
        x[i // 4, 0, 32 * (i % 4): 32 * (i % 4) + 32] = torch.ldexp(steps, torch.tensor(e))
    x = x.to(dtype).cuda()
    x = torch.where(torch.isfinite(x), x, torch.zeros_like(x))
    case = ref.Case(zc, fmt, 128, 16, 1, [rows], [rows])
    zc.kv_append(case.cache, case.batch, x, -x)
    e, s = ref.quantize(x, fmt)
    page, token = (t.cuda() for t in case.token_slots(0))
    assert torch.equal(case.cache.k_scales[page, :, token], s)
    assert torch.equal(case.cache.k_elems[page, :, token], e)
    assert torch.equal(case.cache.v_elems[page, :, token], e ^ (0x88 if fmt == zc.FMT_FP4_E2M1 else 0x80))


@pytest.mark.parametrize("fmt", FORMATS)
def test_not_finite(fmt):
    case = ref.Case(zc, fmt, 64, 16, 1, [3], [3])
    x = torch.ones((3, 1, 64), device="cuda")
    x[0, 0, 5], x[1, 0, 40], x[2, 0, 0] = math.nan, math.inf, -math.inf
    zc.kv_append(case.cache, case.batch, x, x)
    out = torch.empty_like(x)
    zc.kv_read(case.cache, case.batch, out, None)
    bad = torch.zeros((3, 1, 64), dtype=torch.bool, device="cuda")
    if fmt == zc.FMT_FP4_E2M1:
        bad[0, 0, :32] = bad[1, 0, 32:] = bad[2, 0, :32] = True
    else:
        bad[0, 0, 5] = bad[1, 0, 40] = bad[2, 0, 0] = True
    assert torch.equal(torch.isnan(out), bad) and bool((out[~bad] == 1).all())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
def test_all_bytes_read(fmt, dtype):
    case = ref.Case(zc, fmt, 128, 64, 2, [640], [640], low=-127)
    case.cache.k_scales[case.table[0, 0].item(), 0, 0, 0] = 255
    out = torch.empty((640, 2, 128), dtype=dtype, device="cuda")
    zc.kv_read(case.cache, case.batch, out, None)
    want = case.tokens(0)[0].transpose(0, 1)
    want = want.float().to(dtype) if dtype != torch.float32 else want.float()
    assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(torch.nan_to_num(out), torch.nan_to_num(want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset,row,head", [(0, 1536, 128), (0, 129, 5 * 129), (3, 400, 131), (8, 1000, 144)])
def test_strides(dtype, offset, row, head):
    # slices of a fused projection's result; heads before rows; odd offsets and pitches
    heads, rows = 2, 5
    case = ref.Case(zc, zc.FMT_FP4_E2M1, 128, 16, heads, [40], [rows])
    whole = numbers((1, 16384), dtype, 3)[0]
    x = torch.as_strided(whole, (rows, heads, 128), (row, head, 1), offset)
    v = torch.as_strided(whole, (rows, heads, 128), (row, head, 1), offset + 4096)
    before = [t.clone() for t in (case.cache.k_elems, case.cache.k_scales)]
    zc.kv_append(case.cache, case.batch, x, v)
    for got, want in zip((case.cache.k_elems, case.cache.k_scales), expected(case, before, x, "k")):
        assert torch.equal(got, want)
    room = torch.full((16384,), 7.0, dtype=dtype, device="cuda")
    out = torch.as_strided(room, (rows, heads, 128), (row, head, 1), offset)
    zc.kv_read(case.cache, case.batch, out, None)
    want = torch.full_like(room, 7.0)
    torch.as_strided(want, (rows, heads, 128), (row, head, 1), offset).copy_(case.tokens(0)[0].transpose(0, 1)[-rows:].to(dtype))
    assert torch.equal(room, want)


def test_many_sequences():
    # more sequences than lanes, and than lanes squared, with empty ones between them
    for seqs in (33, 1500):
        lens = [(7 * b) % 23 for b in range(seqs)]
        new = [min(n, b % 3) for b, n in enumerate(lens)]
        case = ref.Case(zc, zc.FMT_FP4_E2M1, 64, 16, 1, lens, new)
        x = numbers((case.rows, 1, 64), torch.bfloat16, 4)
        before = [t.clone() for t in (case.cache.v_elems, case.cache.v_scales)]
        zc.kv_append(case.cache, case.batch, x, x)
        e, s = ref.quantize(x, case.fmt)
        want_e, want_s = (t.cpu() for t in before)
        for b, n in enumerate(new):
            for j in range(n):
                t = lens[b] - n + j
                want_e[case.table[b, t // 16], :, t % 16], want_s[case.table[b, t // 16], :, t % 16] = e[case.first_list[b] + j].cpu(), s[case.first_list[b] + j].cpu()
        assert torch.equal(case.cache.v_elems.cpu(), want_e) and torch.equal(case.cache.v_scales.cpu(), want_s)


def test_bad_pages_and_lengths_are_not_followed():
    case = ref.Case(zc, zc.FMT_FP4_E2M1, 64, 16, 2, [40, 20, 16], [40, 20, 16])
    case.batch.page_table[0, 1], case.batch.page_table[1, 0] = 1 << 30, -5
    x = numbers((case.rows, 2, 64), torch.bfloat16, 5)
    before = [t.clone() for t in (case.cache.k_elems, case.cache.k_scales)]
    zc.kv_append(case.cache, case.batch, x, x)
    assert zc.kv_status() == zc.E_CORRUPT and zc.kv_status() == zc.OK
    want = expected(case, before, x, "k")
    for place, b in ((1, 0), (0, 1)):
        page = case.table[b, place]
        for w, o in zip(want, before):
            w[page] = o[page]
    for got, w in zip((case.cache.k_elems, case.cache.k_scales), want):
        assert torch.equal(got, w)
    out = torch.full_like(x, 7.0)
    zc.kv_read(case.cache, case.batch, out, None)
    assert zc.kv_status() == zc.E_CORRUPT
    assert bool((out[16:32] == 0).all()) and bool((out[40:56] == 0).all()) and not bool((out == 7.0).any())
    # a length below 0 is 0; one above the table's room is that
    case.batch.page_table.copy_(case.table.clamp(min=0))
    case.batch.lens[0], case.batch.lens[2] = -1, 1 << 30
    zc.kv_read(case.cache, case.batch, out, None)
    assert zc.kv_status() == zc.E_CORRUPT
    assert bool((out[:40] == 0).all())


def test_captured_calls_follow_lengths():
    case = ref.Case(zc, zc.FMT_FP8_E4M3, 64, 16, 2, [20, 5], [1, 1])
    x = numbers((2, 2, 64), torch.bfloat16, 6)
    out = torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            zc.kv_append(case.cache, case.batch, x, x)
            zc.kv_read(case.cache, case.batch, None, out)
    for step in range(3):
        case.batch.lens.copy_(torch.tensor([21 + step, 6 + step], dtype=torch.int32))
        x.copy_(numbers((2, 2, 64), torch.bfloat16, 7 + step))
        graph.replay()
        torch.cuda.synchronize()
        case.lens_list = [21 + step, 6 + step]
        for b in range(2):
            assert torch.equal(out[b].double(), case.tokens(b)[1][:, -1])
        assert torch.equal(out.double(), ref.values(*ref.quantize(x, case.fmt), case.fmt))
