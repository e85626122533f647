"""Operators on a quantised key/value cache at the ends of their ranges, and attention whose waits run out."""
import contextlib
import math

import pytest
import torch

import kv_reference as ref
from paper_2508_19263_b200 import binding as zc
from test_gpu_kv_attention import BF16, E4M3, F16, FP4, check, clean, queries, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


@contextlib.contextmanager
def stalled(stall):
    try:
        zc.test_set_wait_limit(1000)
        stall(True)
        yield
    finally:
        zc.test_set_wait_limit(0)
        stall(False)


# copies that nobody starts (few rows); matrix instructions that nobody starts (many rows)
@pytest.mark.parametrize("fmt,dim", [(FP4, 128), (E4M3, 64)])
@pytest.mark.parametrize("stall,new", [(zc.test_stall_decoder, [1, 1, 1]), (zc.test_stall_decoder, [5, 1, 3]), (zc.test_stall_math, [100, 64, 33])])
def test_waits_that_run_out(fmt, dim, stall, new):
    case = ref.Case(zc, fmt, dim, 16, 4, [3000, 65, 700], new)
    q = queries(case, 4, BF16)
    ws = workspace(case, 16)
    want = zc.kv_attention(case.cache, case.batch, q, torch.empty_like(q), ws)
    out = torch.empty_like(q)
    assert zc.kv_status() == zc.OK
    with stalled(stall):
        for _ in range(3):
            zc.kv_attention(case.cache, case.batch, q, out, ws)
        assert zc.kv_status() == zc.E_DEVICE_TIMEOUT
    assert zc.kv_status() == zc.OK
    zc.kv_attention(case.cache, case.batch, q, out, ws)
    assert zc.kv_status() == zc.OK and torch.equal(out, want)


@pytest.mark.parametrize("new", [1, 3, 40])
def test_a_long_sequence(new):
    case = ref.Case(zc, FP4, 64, 128, 1, [70001], [new])
    check(case, queries(case, 2, F16))


@pytest.mark.parametrize("fmt", [FP4, E4M3])
@pytest.mark.parametrize("most_new", [1, 3, 70])
def test_many_sequences(fmt, most_new):
    # more than 32: the runs' places are looked for in two steps; empty sequences, sequences without rows
    lens = [(37 * b) % 211 for b in range(131)]
    new = [0 if b % 7 == 3 else min(n, 1 + (b * 5) % most_new) for b, n in enumerate(lens)]
    case = ref.Case(zc, fmt, 64, 32, 2, lens, new)
    check(case, queries(case, 3, BF16))


def test_the_most_sequences():
    case = ref.Case(zc, FP4, 64, 16, 1, [b % 40 for b in range(4096)], [1 if b % 40 else 0 for b in range(4096)])
    q = queries(case, 1, BF16)
    out = torch.empty_like(q)
    zc.kv_attention(case.cache, case.batch, q, out, workspace(case, 1))
    for b in range(0, 4096, 61):
        if case.new[b]:
            k, v = case.tokens(b)
            r = case.first_list[b]
            want = torch.softmax(q[r, 0].double() @ k[0].t() / 8, 0) @ v[0]
            assert bool(((out[r, 0].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -10 * v[0].abs().amax(0)).all())


def test_offsets_beyond_32_bits():
    # keys and values of 5.9 GB each; a sequence in the last pages, one in the first
    pages, heads = 90000, 8
    cache = zc.KvCache(*[torch.zeros((pages, heads, 64, w), dtype=torch.uint8, device="cuda") for w in (128, 4, 128, 4)], E4M3)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    batch = zc.KvBatch(i32([[pages - 1, pages - 3], [0, 70000]]), i32([100, 128]), i32([0, 100, 228]), 128)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((228, heads, 128), generator=g, device="cuda").to(BF16) for _ in range(2))
    zc.kv_append(cache, batch, k, v)
    back = zc.kv_read(cache, batch, torch.empty_like(k), torch.empty_like(v))
    values = [ref.values(*ref.quantize(t, E4M3), E4M3) for t in (k, v)]
    assert all(torch.equal(b.double(), x) for b, x in zip(back, values))
    for n in (1, 40):
        one = zc.KvBatch(batch.page_table, batch.lens, i32([0, n, 2 * n]), n)
        q = torch.randn((2 * n, heads, 128), generator=g, device="cuda").to(BF16)
        out = zc.kv_attention(cache, one, q, torch.empty_like(q), torch.empty(zc.kv_attention_workspace_bytes(cache, one, heads), dtype=torch.uint8, device="cuda"), causal=False)
        for b, r in ((0, slice(0, 100)), (1, slice(100, 228))):
            x = torch.einsum("rhd,thd->hrt", q[b * n: b * n + n].double(), values[0][r]) * 128 ** -0.5
            want = torch.einsum("hrt,thd->rhd", torch.softmax(x, -1), values[1][r])
            assert bool(((out[b * n: b * n + n].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -10 * values[1][r].abs().amax(0)).all())


def test_nothing_cached():
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    for pages, table in ((0, i32([]).reshape(2, 0)), (0, i32([[5], [6]])), (3, i32([]).reshape(2, 0))):
        cache = zc.kv_empty(pages, 2, 16, 64)
        for first in ([0, 1, 2], [0, 40, 41]):
            batch = zc.KvBatch(table, i32([0, 0]), i32(first), first[1])
            q = torch.ones((first[-1], 4, 64), dtype=BF16, device="cuda")
            out, lse = torch.full_like(q, 7.0), torch.zeros((first[-1], 4), device="cuda")
            ws = torch.empty(zc.kv_attention_workspace_bytes(cache, batch, 4), dtype=torch.uint8, device="cuda")
            for causal in (True, False):
                zc.kv_attention(cache, batch, q, out, ws, causal=causal, d_lse=lse)
                assert bool((out == 0).all()) and bool((lse == -math.inf).all())
            zc.kv_append(cache, batch, q[:, :2], q[:, :2])
            zc.kv_read(cache, batch, out[:, :2].fill_(7.0), None)
            assert bool((out[:, :2] == 0).all())
    # pages in a table of a cache without any are not followed
    batch = zc.KvBatch(i32([[0]]), i32([5]), i32([0, 1]), 1)
    cache = zc.kv_empty(0, 2, 16, 64)
    q = torch.ones((1, 4, 64), dtype=BF16, device="cuda")
    out = zc.kv_attention(cache, batch, q, torch.empty_like(q), torch.empty(zc.kv_attention_workspace_bytes(cache, batch, 4), dtype=torch.uint8, device="cuda"))
    assert zc.kv_status() == zc.E_CORRUPT and bool((out == 0).all())


@pytest.mark.parametrize("new", [[1, 1], [4, 60]])
def test_sequences_that_share_pages(new):
    # a common beginning; each sequence's own tokens behind it
    case = ref.Case(zc, FP4, 128, 16, 2, [200, 170], new)
    case.table[1, :9] = case.table[0, :9]
    case.batch.page_table.copy_(case.table)
    check(case, queries(case, 4, BF16))


@pytest.mark.parametrize("new", [1, 80])
def test_two_streams_at_once(new):
    # calls that overlap, each with a workspace of its own
    case = ref.Case(zc, FP4, 128, 16, 4, [2000, 900], [new, new])
    q = queries(case, 4, BF16)
    want = zc.kv_attention(case.cache, case.batch, q, torch.empty_like(q), workspace(case, 16))
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs, spaces = [torch.empty_like(q) for _ in streams], [workspace(case, 16) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, o, w in zip(streams, outs, spaces):
            zc.kv_attention(case.cache, case.batch, q, o, w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("new", [1, 80])
def test_two_graphs_that_share_a_workspace(new):
    case = ref.Case(zc, E4M3, 64, 32, 2, [700, 100], [new, 1])
    q, ws = [queries(case, 4, BF16, seed) for seed in (1, 2)], workspace(case, 8)
    want = [zc.kv_attention(case.cache, case.batch, x, torch.empty_like(x), ws).clone() for x in q]
    outs, graphs, s = [torch.empty_like(x) for x in q], [], torch.cuda.Stream()
    torch.cuda.synchronize()
    for x, o in zip(q, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=s):
            zc.kv_attention(case.cache, case.batch, x, o, ws)
    for order in ((0, 1), (1, 0), (0, 0, 1)):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for k in order:
                graphs[k].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


@pytest.mark.parametrize("new", [1, 70])
def test_nan_in_values(new):
    # a value's scale, seen by some rows of a tile only; the others' results stay as they are
    for fmt in (FP4, E4M3):
        case = ref.Case(zc, fmt, 64, 16, 1, [100], [new])
        q = queries(case, 2, BF16)
        ws = workspace(case, 2)
        want = zc.kv_attention(case.cache, case.batch, q, torch.empty_like(q), ws).clone()
        for place in (19, 60):
            page = case.table[0, place // 16].item()
            kept = case.cache.v_scales[page, 0, place % 16, 1].item()
            case.cache.v_scales[page, 0, place % 16, 1] = 255
            got = zc.kv_attention(case.cache, case.batch, q, torch.empty_like(q), ws)
            case.cache.v_scales[page, 0, place % 16, 1] = kept
            sees = (torch.arange(100 - new, 100) >= place).cuda()
            assert bool(torch.isnan(got[sees][..., 32:]).all()) and torch.equal(got[~sees], want[~sees])
