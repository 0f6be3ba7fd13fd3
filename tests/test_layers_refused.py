"""Calls for one layer's cache refuse the caches of all layers as they refuse other misuse."""
import copy

import pytest
import torch

from paper_2511_18871_amd import binding as B


def test_a_call_for_one_layer_refuses_all_layers():
    k = torch.zeros(2, 4, 2, 16, 64)
    layers, i32 = B.KvLayers(k, k.clone()), lambda *s: torch.zeros(*s, dtype=torch.int32)
    for call in (lambda: B.sp_attn_decode(layers, torch.zeros(1, 2, 64), None, None, None, i32(1, 1), i32(1), 0.1),
                 lambda: B.sp_attn_tree_decode(layers, torch.zeros(3, 4, 64), None, [3], None, None, None, i32(1, 2), i32(1), 0.1),
                 lambda: B.sp_attn_tree_decode(layers, torch.zeros(3, 64), None, [3], None, None, None, i32(1, 2), i32(1), 0.1),
                 lambda: B.sp_attn_cache_append(layers, torch.zeros(1, 2, 64), torch.zeros(1, 2, 64), i32(1, 1), i32(1), 1e4)):
        with pytest.raises(B.SpAttnError, match="one layer") as e:
            call()
        assert e.value.status == B.SP_ERR_INVALID_ARG
    assert not hasattr(layers, "head_dim") and not hasattr(layers, "anything") and len(layers) == 2
    with pytest.raises(AttributeError, match="anything"):
        layers.anything
    assert torch.equal(copy.copy(layers).k, k)
