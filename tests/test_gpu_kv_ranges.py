"""Attention over a quantised key/value cache at the ends of FP32's range, and what it does not touch."""
import math

import pytest
import torch

import kv_reference as ref
from paper_2508_19263_b200 import binding as zc
from test_gpu_kv_attention import BF16, E4M3, F16, FP4, check, clean, queries, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


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
