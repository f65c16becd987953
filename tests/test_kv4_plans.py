"""Sizes of the attention over the 4-bit cache that its contract allows have a plan (no GPU needed)."""
import pytest

import paper_2609_30846_gb300 as ip


@pytest.mark.parametrize("B,T,H,Hkv,max_len", [
    (64, 2048, 32, 8, 1 << 20), (64, 2048, 32, 8, 1 << 28), (65535, 1, 8, 8, 1 << 20), (65535, 1, 64, 8, 1 << 28),
    (1, 2048, 8200, 1, 3), (1, 2048, 65535, 1, 1 << 28), (2048, 1, 64, 64, 1 << 28), (1, 1, 65535, 65535, 1 << 28),
    (20000, 2048, 8, 8, 100)])
def test_allowed_sizes_have_a_plan(B, T, H, Hkv, max_len):
    assert 256 <= ip.kv4_attention_workspace_bytes(B, T, H, Hkv, max_len) <= 1 << 23


@pytest.mark.parametrize("sizes", [(65535, 2048, 65535, 65535, 10), (65535, 2048, 1024, 1024, 10)])
def test_more_items_than_a_grid_holds_have_none(sizes):
    with pytest.raises(ip.IpError):
        ip.kv4_attention_workspace_bytes(*sizes)
