"""What the errors of the operators on FP8 matrices say."""
import pytest
import torch

from paper_2508_19263_b200 import binding as zc


def test_too_large_speaks_of_sizes():
    # 65 tokens, refused before anything reaches a GPU: no built-in scratch is concerned
    m = zc.Fp8MoeLayer(torch.zeros((4, 64), dtype=torch.bfloat16), *(torch.zeros(s, dtype=torch.uint8) for s in ((4, 2, 32, 64), (4, 2, 1, 1), (4, 64, 32), (4, 1, 1))), 2)
    status = zc._lib.zc_fp8_moe(m._ref, 65, 1 << 25, 64, 1 << 26, 64, None, None, 1 << 27, 1 << 30, None)
    assert status == zc.E_TOO_LARGE
    with pytest.raises(zc.ZcError, match="size is above what the call takes"):
        raise zc.ZcError(status, "zc_fp8_moe")
