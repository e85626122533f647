"""A mixture-of-experts layer of one expert: its router is a single row, which has no pitch, whatever its length."""
import pytest
import torch

from paper_2508_19263_b200 import binding as zc

HIDDEN, INTER = 513, 40


def layer(router, seed=101):
    g = torch.Generator().manual_seed(seed)
    pad = lambda t: torch.nn.functional.pad(t, (0, -t.shape[-1] % 16))[..., : t.shape[-1]]  # noqa: E731
    elems = lambda *s: pad((torch.randint(0, 256, s, generator=g, dtype=torch.uint8) & 0xBF).to(router.device))  # noqa: E731
    scales = lambda *s: torch.full(s, 120, dtype=torch.uint8, device=router.device)  # noqa: E731
    return zc.Fp8MoeLayer(router, elems(1, 2, INTER, HIDDEN), scales(1, 2, 1, 5), elems(1, HIDDEN, INTER), scales(1, 5, 1), 1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_router_of_one_odd_row_is_taken(dtype):
    m = layer(torch.zeros((1, HIDDEN), dtype=dtype))
    assert m.desc.ld_router == 520 and m.workspace_bytes(3) > 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_its_results_are_those_of_a_padded_row(dtype):
    g = torch.Generator(device="cuda").manual_seed(102)
    wide = torch.full((1, 520), float("nan"), dtype=dtype, device="cuda")
    wide[:, :HIDDEN] = torch.randn((1, HIDDEN), generator=g, device="cuda")
    x = torch.nn.functional.pad(torch.randn((5, HIDDEN), generator=g, device="cuda").to(dtype), (0, 7))[:, :HIDDEN]
    got = []
    for router in (wide[:, :HIDDEN].contiguous(), wide[:, :HIDDEN]):
        m, weights = layer(router), torch.empty((5, 1), device="cuda")
        got.append(zc.fp8_moe(m, x, torch.empty((5, HIDDEN), dtype=dtype, device="cuda"), torch.empty(m.workspace_bytes(5), dtype=torch.uint8, device="cuda"), d_weights=weights))
        assert bool((weights == 1).all())                                    # one expert: the softmax of one logit
    assert torch.equal(got[0], got[1]) and bool(torch.isfinite(got[0]).all()) and bool(got[0].any())
    assert zc.fp8_status() == zc.OK
