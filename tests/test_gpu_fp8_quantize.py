"""zc_fp8_quantize at sizes whose thread numbers do not fit into 32 bits."""
import numpy as np
import pytest
import torch

import fp8_reference as ref
from paper_2508_19263_b200 import binding as zc

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_more_blocks_than_32_bits_of_threads():
    # eight lanes a block of 1 x 128: 2^29 blocks have 2^32 lanes.  Rows of one element, 10 GB in all
    rows, tail = (1 << 29) + 40, 300
    x = torch.zeros((rows, 1), dtype=torch.bfloat16, device=DEV)
    x[-tail:] = torch.randn((tail, 1), generator=torch.Generator(device=DEV).manual_seed(51), device=DEV).bfloat16()
    q = zc.fp8_empty(rows, 1)
    q.elems.fill_(0xAB)
    q.scales.fill_(0xAB)
    zc.fp8_quantize(x, q)
    elems, scales, _ = ref.quantize(x[-tail:].double().cpu().numpy(), zc.FMT_FP8_E4M3, 1)
    assert np.array_equal(q.elems[-tail:].cpu().numpy(), elems) and np.array_equal(q.scales[-tail:].cpu().numpy(), scales)
    for part in range(0, rows - tail, 1 << 26):                              # zeros everywhere else
        end = min(part + (1 << 26), rows - tail)
        assert not bool(q.elems[part:end].any()) and not bool(q.scales[part:end].any())
