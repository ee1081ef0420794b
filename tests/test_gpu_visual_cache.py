"""The example that takes images through merge, cache, prune, fork and decode, against dense attention."""
import pytest
import torch

pytestmark = pytest.mark.gpu


# the dense form sees the unrounded values of the same rows: bf16 rows round the output (2^-9 rms), an 8-bit cache every
# element of K and V by up to 1/16 (a quarter of that rms, once through the scores and once through the values)
@pytest.mark.parametrize("cache,bound", [("bf16", 2.0 ** -8), ("f32", 2.0 ** -18), ("e4m3", 2.0 ** -4)])
def test_images_to_answers(cache, bound):
    import sys, os                                                                      # noqa: E401
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import visual_cache

    assert torch.cuda.is_available()
    r = visual_cache.run(3, 2, 20, cache)
    assert r["cached_tokens"] == 6 * (9 + 36 + 17 + 20)
    # each image's full pages once, and the tail and the new tokens of each question
    assert r["pages_used"] == 3 * 3 + 6 * 3
    assert r["relative_error"] <= bound
