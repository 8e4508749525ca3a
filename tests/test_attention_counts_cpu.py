"""Counts that an int32 cannot hold are refused by name: the C entry points would see them
cut to 32 bits (no GPU needed)."""
import pytest
import torch

from paper_2607_00466_amd import binding as B


def d(**changes):
    return B.attn_dims(**(dict(R=4, Hq=8, Hkv=2, D=128, block_size=16, max_blocks=8, num_blocks=64) | changes))


@pytest.mark.parametrize("name,value", [("window", 1 << 32), ("window", (1 << 32) + 5), ("window", -1 - (1 << 32))])
def test_window(name, value):
    t = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match=name):
        B.moe_attn_decode(t, t, t, t, t, d(), t, t, t, window=value)


@pytest.mark.parametrize("name,values", [("budget", (16 + (1 << 32), 4)), ("recent", (16, 1 << 32)), ("recent", (16, 1 << 31))])
def test_budget_and_recent(name, values):
    t = torch.zeros(4, 8, 128)
    with pytest.raises(ValueError, match=name):
        B.moe_kv_evict(t, t, t, t, t, d(), *values, t, t, t, t, t, t)


@pytest.mark.parametrize("name", ["R", "Hq", "Hkv", "D", "block_size", "max_blocks", "num_blocks"])
def test_dims(name):
    with pytest.raises(ValueError, match=name):
        d(**{name: (1 << 32) + 4})
