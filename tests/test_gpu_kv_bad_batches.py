"""Lengths and first rows outside their ranges: what the calls on a quantised key/value cache do with them, and that sequences beside them are not disturbed."""
import math

import pytest
import torch

import kv_reference as ref
from paper_2508_19263_b200 import binding as zc
from test_gpu_kv_attention import BF16, FP4, clean, queries, workspace  # noqa: F401

pytestmark = pytest.mark.gpu
LENS, NEW = [40, 90, 64], [5, 70, 9]
FIRST = [0, 5, 75, 84]
ROWS = 84


def batch_of(case, lens, first, max_new):
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return zc.KvBatch(case.batch.page_table, i32(lens), i32(first), max_new)


def attend(case, batch, q, causal=True):
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    ws = torch.randint(0, 256, (zc.kv_attention_workspace_bytes(case.cache, batch, q.shape[1]),), dtype=torch.uint8, device="cuda")
    zc.kv_attention(case.cache, batch, q, out, ws, causal=causal, d_lse=lse)
    return out, lse


def compare(case, q, out, lse, first, new, lens):
    """Rows of sequences with new > 0 are the formula's, all others untouched; rows that two of them have, since the first rows fall, have something of either."""
    right = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    mine = torch.zeros(len(q), dtype=torch.int32, device="cuda")
    for b, n in enumerate(new):
        case.first_list, case.new, case.lens_list = list(first), [n if c == b else 0 for c in range(len(new))], list(lens)
        want, want_lse, bound = ref.attention(case, q, case.dim ** -0.5)
        rows = slice(first[b], first[b] + n)
        mine[rows] += 1
        ok = ((out.double() - want).abs() <= ref.tolerance(want, bound, q.dtype)).all(-1)
        none = torch.isinf(want_lse)
        ok &= torch.where(none, (lse == -math.inf) & (out == 0).all(-1), (lse.double() - want_lse).abs() <= 2.0 ** -10)
        right[rows] |= ok[rows]
    assert bool((right.all(-1) | (mine != 1)).all())
    assert bool((out[mine == 0] == 7.0).all()) and bool((lse[mine == 0] == 7.0).all())


def make():
    case = ref.Case(zc, FP4, 64, 16, 2, LENS, NEW)
    case.batch.page_table.clamp_(min=0)
    case.table = case.batch.page_table.cpu()
    return case


# (first rows, rows that sequences then have): those of a sequence that do not lie within the call's rows, or go backwards, are none
@pytest.mark.parametrize("first,new", [
    ([0, 5, 1 << 30, 84], [5, 0, 0]), ([-(1 << 31), 5, 75, 84], [0, 70, 9]), ([0, 5, 75, (1 << 31) - 1], [5, 70, 0]), ([0, 5, 75, ROWS + 1], [5, 70, 0]), ([-1, 5, 75, 84], [0, 70, 9]),
    ([60, 30, 75, 84], [0, 45, 9]), ([80, 70, 60, 50], [0, 0, 0]), ([0, 5, 3, 84], [5, 0, 81])])
@pytest.mark.parametrize("max_new", [1, 81])
def test_first_rows(first, new, max_new):
    case = make()
    q = queries(case, 4, BF16)
    batch = batch_of(case, LENS, first, max_new)
    out, lse = attend(case, batch, q)
    assert zc.kv_status() == zc.E_CORRUPT and zc.kv_status() == zc.OK
    compare(case, q, out, lse, [max(0, min(f, ROWS)) for f in first[:3]], new, LENS)


@pytest.mark.parametrize("lens,counts", [([-3, 90, 64], [0, 90, 64]), ([40, -(1 << 31), 64], [40, 0, 64]), ([40, 90, (1 << 31) - 1], [40, 90, 96]), ([97, 90, 64], [96, 90, 64]), ([-1, 1 << 30, -1], [0, 96, 0])])
@pytest.mark.parametrize("max_new", [1, 70])
def test_lengths(lens, counts, max_new):
    case = make()
    assert case.table.shape[1] * 16 == 96                         # what a row of the table has room for
    q = queries(case, 4, BF16)
    batch = batch_of(case, lens, FIRST, max_new)
    out, lse = attend(case, batch, q)
    assert zc.kv_status() == zc.E_CORRUPT and zc.kv_status() == zc.OK
    compare(case, q, out, lse, FIRST, NEW, counts)
    # the same with the lengths that they count as
    case.new = list(NEW)
    again = attend(case, batch_of(case, counts, FIRST, max_new), q)
    assert zc.kv_status() == zc.OK and torch.equal(again[0], out) and torch.equal(again[1], lse)
    # reading: rows that have no place are zeros, the others those tokens
    got = torch.full((ROWS, 2, 64), 7.0, device="cuda")
    zc.kv_read(case.cache, batch, got, None)
    assert zc.kv_status() == zc.E_CORRUPT
    case.lens_list = counts
    want = torch.zeros_like(got)
    for b, n in enumerate(NEW):
        have = min(n, counts[b])
        want[FIRST[b + 1] - have: FIRST[b + 1]] = case.tokens(b)[0].transpose(0, 1)[counts[b] - have: counts[b]].float()
    assert torch.equal(got, want)
    # writing: nothing but those rows' places
    before = case.cache.k_elems.clone()
    zc.kv_append(case.cache, batch, torch.ones_like(got), torch.ones_like(got))
    assert zc.kv_status() == zc.E_CORRUPT
    free = torch.ones(before.shape[:3], dtype=torch.bool)
    for b, n in enumerate(NEW):
        page, token = case.token_slots(b)
        have = min(n, counts[b])
        free[page[counts[b] - have:], :, token[counts[b] - have:]] = False
    assert torch.equal(case.cache.k_elems[free.cuda()], before[free.cuda()])
