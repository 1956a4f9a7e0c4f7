"""Kv8.empty: what it refuses (no GPU needed)."""
import pytest
import torch


@pytest.mark.parametrize("capacity,block,dtype", [(64, 0, torch.int8), (64, -32, torch.int8), (0, 32, torch.int8), (-5, 32, torch.int8), (64, 32, torch.bfloat16)])
def test_refusals(capacity, block, dtype):
    import paper_2411_05787_amd as rk
    with pytest.raises(ValueError, match="capacity"):
        rk.Kv8.empty(rk.Geom(1, 4, 2, 128, 0.1), capacity, block, dtype, device="cpu")
