"""Kernels on FP8 matrices whose waits run out while their copies are under way: they wait for these before they return, report, and leave
nothing behind for the next call."""
import contextlib

import pytest
import torch

from paper_2508_19263_b200 import binding as zc

pytestmark = pytest.mark.gpu
DEV = "cuda"
GAVE_UP, SETTLED = 1, 2                                                      # 4: something was still under way at the end


@contextlib.contextmanager
def stalled(stall):
    """Copies are started but no matrix instruction, or no copies, so that waits run out."""
    try:
        zc.test_set_wait_limit(1000)
        stall(True)
        yield
    finally:
        zc.test_set_wait_limit(0)
        stall(False)


# one block, several parts of k, one tile a block; pairs of blocks with fewer steps than stages, with more, with several tiles a pair
@pytest.mark.parametrize("m,n,k", [(1, 128, 128), (1, 256, 4096), (64, 512, 2048), (300, 400, 640), (1600, 1792, 128), (1600, 1792, 512), (1601, 1795, 2050), (2600, 2400, 768)])
@pytest.mark.parametrize("stall", [zc.test_stall_math, zc.test_stall_decoder])
def test_products(m, n, k, stall):
    g = torch.Generator(device=DEV).manual_seed(91)
    a, b = (zc.fp8_quantize(torch.randn((r, k), generator=g, device=DEV), zc.fp8_empty(r, k)) for r in (m, n))
    want = zc.fp8_matmul(a, b, torch.empty((m, n), device=DEV))
    d = torch.empty_like(want)
    assert zc.fp8_status() == zc.OK and zc.test_fp8_marks() == 0
    with stalled(stall):
        for _ in range(3):
            zc.fp8_matmul(a, b, d)
        assert zc.fp8_status() == zc.E_DEVICE_TIMEOUT
        assert zc.test_fp8_marks() == GAVE_UP | SETTLED
    zc.fp8_matmul(a, b, d)
    assert zc.fp8_status() == zc.OK and torch.equal(d, want)


@pytest.mark.parametrize("tokens", [1, 12, 64])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("stall", [zc.test_stall_math, zc.test_stall_decoder])
def test_layers(tokens, dtype, stall):
    experts, hidden, inter = 16, 1100, 600
    g = torch.Generator(device=DEV).manual_seed(92)
    elems = lambda *s: (torch.randint(0, 256, s, generator=g, device=DEV, dtype=torch.uint8) & 0xBF)  # noqa: E731
    scales = lambda *s: torch.full(s, 120, dtype=torch.uint8, device=DEV)  # noqa: E731
    pad = lambda t: torch.nn.functional.pad(t, (0, -t.shape[-1] % 16))[..., : t.shape[-1]]  # noqa: E731
    layer = zc.Fp8MoeLayer(torch.nn.functional.pad(torch.randn((experts, hidden), generator=g, device=DEV).to(dtype), (0, 4))[:, :hidden],
                           pad(elems(experts, 2, inter, hidden)), scales(experts, 2, 5, 9), pad(elems(experts, hidden, inter)), scales(experts, 9, 5), 4)
    x = torch.nn.functional.pad(torch.randn((tokens, hidden), generator=g, device=DEV).to(dtype), (0, 4))[:, :hidden]
    ws = torch.empty(layer.workspace_bytes(tokens), dtype=torch.uint8, device=DEV)
    want = zc.fp8_moe(layer, x, torch.empty((tokens, hidden), dtype=dtype, device=DEV), ws)
    y = torch.empty_like(want)
    assert zc.fp8_status() == zc.OK and zc.test_fp8_marks() == 0 and bool(torch.isfinite(want).all())
    with stalled(stall):
        for _ in range(3):
            zc.fp8_moe(layer, x, y, ws)
        assert zc.fp8_status() == zc.E_DEVICE_TIMEOUT
        assert zc.test_fp8_marks() == GAVE_UP | SETTLED
    zc.fp8_moe(layer, x, y, ws)
    assert zc.fp8_status() == zc.OK and torch.equal(y, want)
