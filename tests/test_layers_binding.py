"""What layers.py refuses before it asks for a device."""
import pytest
import torch

from paper_1503_02852_amd import RnnError, layers

WIDE = (1 << 32) + 8      # 8, if cut to 32 bits


@pytest.mark.parametrize("name", ["T", "N", "heads", "kv_heads", "dim_k", "dim_v"])
def test_attention_sizes_beyond_32_bits(name):
    sizes = dict(T=8, N=8, heads=8, kv_heads=8, dim_k=8, dim_v=8)
    with pytest.raises(RnnError, match=name):
        layers.LinearAttention(**dict(sizes, **{name: WIDE}))


def test_rows_beyond_32_bits():
    with pytest.raises(RnnError, match="dim"):
        layers.AddNorm(1, WIDE)
    x = torch.empty(WIDE, dtype=torch.bfloat16, device="meta")
    with pytest.raises(RnnError, match="dim"):
        layers.dropout(x, x, 0.5, 1)
