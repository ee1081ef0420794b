"""In the example of questions about merged images a merged token's size counts once: in the values that enter the cache, or in the scores."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_sizes_count_once(monkeypatch):
    import visual_question
    luvc = visual_question.luvc

    seen = {}

    def watch(name, argument):
        call = getattr(luvc, name)

        def watched(*args, **named):
            seen.setdefault(name, []).append(named.get(argument))
            return call(*args, **named)
        monkeypatch.setattr(luvc, name, watched)

    watch("kv_write", "sizes")
    watch("attn_cross", "key_bias")
    watch("attn_decode", "key_bias")
    r = visual_question.run(2, 5, 4)
    (sizes,), (cross,), (decode,) = seen["kv_write"], seen["attn_cross"], seen["attn_decode"]
    assert (sizes is None) == (cross is not None) == (decode is not None)
    assert torch.isfinite(torch.tensor([r["cross_error"], r["decode_error"], r["cache_error"]])).all()
