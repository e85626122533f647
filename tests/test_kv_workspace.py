"""Workspaces that are not the memory that their size says."""
import pytest
import torch

from paper_2508_19263_b200 import binding as zc


@pytest.mark.parametrize("space", [torch.zeros(1, dtype=torch.uint8).expand(1 << 24), torch.zeros(1 << 12, dtype=torch.uint8)[::2], torch.zeros((64, 64), dtype=torch.uint8).t()])
def test_workspaces_with_gaps_or_without_memory_are_refused(space):
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    x = torch.zeros((1, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="contiguous"):
        zc.kv_attention(zc.kv_empty(4, 2, 16, 64, device="cpu"), zc.KvBatch(i32(0, 1).reshape(1, 2), i32(20), i32(0, 1)), x, torch.empty_like(x), space)
