"""Attention to an encoder's states at the ends of the range: values whose sums are beyond it while their means are inside, and small ones.
The bounds are those of test_gpu_attn_cross."""
import math

import pytest
import torch

from test_gpu_attn_cross import check, inputs, ints, luvc  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("queries,keys", [([300], [500]), ([40, 3], [500, 70]), ([3], [500]), ([150], [20000]), ([17], [30001])])
def test_means_of_large_values_are_in_range(luvc, dtype, D, queries, keys):  # noqa: F811
    q, k, v, qs, ks = inputs(dtype, 4, 2, D, queries, keys, seed=D)
    k.mul_(0.25)
    bias = torch.randn(k.shape[0], generator=torch.Generator().manual_seed(1)).cuda()
    for case in range(3):
        if case == 0:
            v.fill_(3e38)
        if case == 1:
            v.copy_(3e38 - 2e38 * torch.rand(v.shape, generator=torch.Generator().manual_seed(2)).cuda())
            v[:, 1] *= -1
        if case == 2:
            v.copy_(1e-30 * torch.randn(v.shape, generator=torch.Generator().manual_seed(3)).cuda())
        for b in (None, bias):
            out, lse = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, key_bias=b, want_lse=True)
            assert luvc.check_status() == 0
            assert bool(out.isfinite().all())
            check(q, k, v, qs, ks, out, lse, bias=b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("queries", [300, 3])
def test_large_values_the_rest_as_the_formula(luvc, dtype, queries):  # noqa: F811
    """The fifth case of test_infinities_and_nan_give_what_the_formula_gives, asked of both types: one head's values are 3e38 throughout."""
    q, k, v, qs, ks = inputs(dtype, 4, 2, 64, [queries], [500], seed=4)
    k.mul_(0.25)
    v[:, 0] = 3e38
    got = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks).double()
    want = float(v[0, 0, 0])
    assert bool(got[:, :2].isfinite().all())
    assert float((got[:, :2] / want - 1).abs().max()) < (2.0 ** -7 if dtype == "bf16" else 2.0 ** -14)       # (500 + 64) 2^-23 at most, in f32


@pytest.mark.parametrize("queries,keys", [(300, 500), (20, 20000)])
def test_infinities_in_f32_with_many_tokens(luvc, queries, keys):  # noqa: F811
    q, k, v, qs, ks = inputs("f32", 2, 1, 64, [queries], [keys], seed=5)
    k.mul_(0.25)
    v[keys // 2, 0, 3], v[7, 0, 5], v[keys - 1, 0, 5] = math.inf, math.inf, -math.inf
    got = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks)
    assert bool((got[..., 3] == math.inf).all()) and bool(got[..., 5].isnan().all())
    rest = [d for d in range(64) if d not in (3, 5)]
    assert bool(got[..., rest].isfinite().all())
