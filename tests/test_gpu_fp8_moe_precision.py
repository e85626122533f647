"""How exactly zc_fp8_moe keeps an expert's hidden vector, where the rounding of its results does not hide it."""
import numpy as np
import pytest
import torch

import fp8_reference as ref
from paper_2508_19263_b200 import binding as zc

pytestmark = pytest.mark.gpu
DEV = "cuda"
ONE, MINUS_ONE = 0x38, 0xB8                                                  # 1 and -1 in E4M3


def run(layer, x):
    y = torch.empty_like(x)
    zc.fp8_moe(layer, x, y, torch.empty(layer.workspace_bytes(x.shape[0]), dtype=torch.uint8, device=DEV))
    assert zc.fp8_status() == zc.OK
    return y


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_differences_of_neighbouring_hidden_values(dtype):
    """One expert, one token.  The hidden values are sorted, and every row of `down` takes the difference of two neighbours, which is some
    hundredth of them: what the result's own rounding, half a step of the difference, leaves of it shows the hidden values' error.

    Sixteen columns of x are not 0, x is a multiple of 2^-6 below 2 and the weights are multiples of 2^-9 below 2, so gate and up are
    multiples of 2^-15 below 2^6: exact in FP32 in any order, and x in pieces of four bits as well.  h = gate / (1 + exp(-gate)) * up:
    2^-22 of exp, half a unit (2^-24) of the sum, the quotient and the product: less than 2^-21.  As a sum of E4M3 pieces: the first leaves
    2^-4 of the value, every other one (four bits and a sign, of what is at most half a step) 2^-5 of that: 2^-19 after four; where the
    rest is held in FP16 after two, 2^-12 of 2^-9; and half of the last piece's smallest step, 2^-10 2^-12 2^s, while the largest of
    128 is above 224 2^s > 2^7 2^s.  The difference: additions of at most 2^-23 of what is added, two of the first pieces, fewer of the others."""
    hidden, inter = 1024, 1024
    g = torch.Generator().manual_seed(41)
    x = torch.zeros((1, hidden), dtype=torch.float64)
    at = torch.randperm(hidden, generator=g)[:16]
    x[0, at] = torch.randint(-127, 128, (16,), generator=g).double() / 64
    gate_up = torch.randint(0, 256, (1, 2, inter, hidden), generator=g, dtype=torch.uint8) & 0xBF
    scales = torch.full((1, 2, 8, 8), 127, dtype=torch.uint8)
    gate, up = (ref.values(gate_up[0, i].numpy(), scales[0, i].numpy(), zc.FMT_FP8_E4M3, 128) @ x[0].numpy() for i in range(2))
    h = gate / (1 + np.exp(-gate)) * up
    order = np.argsort(h)
    down = torch.zeros((1, hidden, inter), dtype=torch.uint8)
    for r in range(inter - 1):
        down[0, r, order[r + 1]], down[0, r, order[r]] = ONE, MINUS_ONE
    layer = zc.Fp8MoeLayer(torch.zeros((1, hidden), dtype=dtype, device=DEV), gate_up.to(DEV), scales.to(DEV), down.to(DEV),
                           torch.full((1, 8, 8), 127, dtype=torch.uint8, device=DEV), 1)
    y = run(layer, x.to(dtype).to(DEV)).double().cpu().numpy()[0, : inter - 1]
    want = np.diff(h[order])
    assert np.median(want / np.abs(h[order][1:])) < 2.0 ** -6                # neighbours: the test would be blind otherwise
    both = np.abs(h[order][1:]) + np.abs(h[order][:-1])
    off = both * (2.0 ** -21 + 2.0 ** -19 + 2.0 ** -21 + 2.0 ** -22) + 2 * 2.0 ** -29 * np.abs(h).max()
    t = torch.finfo(dtype)
    assert (np.abs(y - want) <= off + t.eps / 2 * (np.abs(want) + off) + t.smallest_normal * t.eps / 2).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_long_sums(dtype):
    """Sums of positive products over 14336 - 128 inner channels, of which the last 128 take all but a trace off again: what is left shows
    what the sums lose on the way, which the rounding of the result would hide otherwise.

    gate is 32, so h = 32 up without a rounding, and up is an element of the weights: h goes into the product exactly.  The accumulators
    cut off what does not fit, less than a unit, 2^-23, of the sum as it is after every 32 columns.  Over the 2048 columns of a part the sum grows
    evenly: (64 + 1) / 2 units of what the part comes to, plus 9.1 / sqrt(2048) of that, six standard deviations of the average of the sums on the way (a
    product of two of the elements deviates by 2.62 times its mean).  All parts come to the whole.  The last four instructions take it off: a unit
    of the whole each.  The parts are added to nearest: half a unit each, and there are seven."""
    hidden, inter, last = 256, 14336, 128
    g = torch.Generator().manual_seed(43)
    values = torch.arange(64, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    x = torch.zeros((1, hidden), dtype=dtype)
    x[0, 0], x[0, 1] = 32.0, 1.0
    gate_up = torch.zeros((1, 2, inter, hidden), dtype=torch.uint8)
    gate_up[0, 0, :, 0] = ONE
    up = torch.randint(0, 64, (inter,), generator=g, dtype=torch.uint8)
    gate_up[0, 1, :, 1] = up
    h = 32 * values[up.long()]
    down = torch.randint(0, 64, (hidden, inter), generator=g, dtype=torch.uint8)
    scales = torch.full((1, 2, inter // 128), 127, dtype=torch.uint8)
    scales[0, :, -1] = 127 + 7                                               # the last block's elements count 128 times
    whole = values[down[:, :-last].long()] @ h[:-last]
    left = whole.clone()
    for c in (inter - last + torch.argsort(h[-last:], descending=True)).tolist():
        code = torch.searchsorted(values, left / (128 * h[c]).clamp(min=1e-9), right=True) - 1      # the largest element that does not take too much
        down[:, c] = code.clamp(0, 63).to(torch.uint8) | 0x80
        left -= values[code.clamp(0, 63)] * 128 * h[c]
    assert bool((left >= 0).all()) and bool((left < 2.0 ** -12 * whole).all())
    layer = zc.Fp8MoeLayer(torch.zeros((1, hidden), dtype=dtype, device=DEV), gate_up.to(DEV), torch.full((1, 2, inter // 128, 2), 127, dtype=torch.uint8, device=DEV),
                           down[None].to(DEV), scales.to(DEV), 1)
    y = run(layer, x.to(DEV)).double().cpu()[0]
    off = whole * 2.0 ** -24 * (65 * (1 + 9.1 / 2048 ** 0.5) + 4 * 2 + 7)
    t = torch.finfo(dtype)
    assert bool(((y - left).abs() <= off + t.eps / 2 * (left + off) + t.smallest_normal * t.eps / 2).all()), ((y - left).abs() / whole * 2.0 ** 24).max()
