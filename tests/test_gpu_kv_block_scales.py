"""Scales that are written along with the rows are the keys' or the values': a cache does not take one memory for both."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_keys_and_values_do_not_share_scales():
    import paper_2512_09010_b200 as luvc

    layers, pages, heads, page, D = 2, 6, 3, 32, 64
    k, v = (torch.zeros((layers, pages, heads, page, D), device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
    at = (layers, pages, heads, page // luvc.KV_BLOCK)
    scale = torch.zeros(at, device="cuda")
    both = torch.zeros((2 * layers - 1,) + at[1:], device="cuda")
    for a, b in ((scale, scale), (scale, scale.view(at)), (both[:layers], both[layers - 1:]), (both[layers - 1:], both[:layers])):
        with pytest.raises(ValueError):
            luvc.KvCache(k, v, 2, 3, k_scale=a, v_scale=b)
    two = torch.zeros((2,) + at, device="cuda")
    assert luvc.KvCache(k, v, 2, 3, k_scale=two[0], v_scale=two[1]).blocks and luvc.KvCache(k, v, 2, 3, k_scale=two[1], v_scale=two[0]).blocks
    heads_only = torch.ones((layers, heads), device="cuda")
    assert not luvc.KvCache(k, v, 2, 3, k_scale=heads_only, v_scale=heads_only).blocks      # (only read)
