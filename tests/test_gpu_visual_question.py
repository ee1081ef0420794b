"""The example that turns, caches, reads back and looks at merged images, against dense attention; and the block-scaled cache in the
example that prunes, forks and decodes."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("images,tokens,heads", [(3, 17, 28), (1, 1, 4), (5, 40, 8)])
def test_questions_about_images(images, tokens, heads):
    import visual_question

    assert torch.cuda.is_available()
    r = visual_question.run(images, tokens, heads)
    assert r["cached_tokens"] == 144 * images
    # weights and results are rounded to bf16 (2^-8 of each at most); decoding rounds the results alone
    assert r["cross_error"] <= 2.0 ** -7 and r["decode_error"] <= 2.0 ** -8
    # e4m3: half a step is 2^-4 of a value at most
    assert r["cache_error"] <= 2.0 ** -4


def test_images_to_answers_in_a_block_scaled_cache():
    import visual_cache

    r = visual_cache.run(3, 2, 20, "e4m3-block")
    assert r["cached_tokens"] == 6 * (9 + 36 + 17 + 20)
    assert r["pages_used"] == 3 * 3 + 6 * 3
    assert r["relative_error"] <= 2.0 ** -4             # every element of K and V by up to 1/16, a quarter of that rms
