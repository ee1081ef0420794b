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


@pytest.mark.parametrize("hq,D,queries,keys", [(2, 64, 700, 16500), (8, 128, 40, 33000), (2, 256, 200, 9000)])
def test_nan_and_infinities_take_no_longer(luvc, hq, D, queries, keys):  # noqa: F811
    """Waits that give up early (a few thousand probes, far more than a tile takes) do not: nothing in the call is worked out at length, once more."""
    q, k, v, qs, ks = inputs("bf16", hq, 1, D, [queries], [keys], seed=6)
    k.mul_(0.25)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    call = lambda: luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, device_status=status)             # noqa: E731
    want = call()
    assert bool(want.isfinite().all()) and luvc.read_status(status) == 0
    assert luvc.lib.luvc_debug_wait_probes(1, 0, status.data_ptr(), stream) == 0
    v[5, 0, 3], v[keys - 1, 0, 7], v[keys // 2, 0, 9], v[11, 0, 9] = math.inf, math.nan, math.inf, -math.inf
    got = call()
    assert luvc.read_status(status) == 0
    assert bool((got[..., 3] == math.inf).all()) and bool(got[..., 7].isnan().all()) and bool(got[..., 9].isnan().all())
    rest = [d for d in range(D) if d not in (3, 7, 9)]
    assert torch.equal(got[..., rest], want[..., rest])
    k[keys // 3, 0, 1] = math.nan
    got = call()
    assert luvc.read_status(status) == 0 and bool(got.isnan().all())
    k[keys // 3, 0, 1], q[queries // 2, 1, 0] = 0.0, math.nan
    got = call()
    assert luvc.read_status(status) == 0
    assert bool(got[queries // 2, 1].isnan().all())
    got[queries // 2, 1] = 0.0
    assert bool(got[..., rest].isfinite().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,heads,D", [(4, 2, 64), (28, 4, 128), (16, 1, 128), (3, 1, 256)])
@pytest.mark.parametrize("queries,keys", [([1], [40000]), ([2], [300]), ([1, 0, 2, 1], [700, 30, 5000, 16]), ([30], [200])])
def test_one_state_of_each_tile_counts(luvc, dtype, hq, heads, D, queries, keys):  # noqa: F811
    """So that every part of a sum is in range, and the parts together are not."""
    q, k, v, qs, ks = inputs(dtype, hq, heads, D, queries, keys, seed=D)
    k.zero_()
    v.fill_(3e38)
    bias = torch.full((k.shape[0],), -math.inf, device="cuda")
    for i, n in enumerate(keys):
        bias[int(ks[i]):int(ks[i]) + n:16] = 0.0
    out, lse = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, key_bias=bias, want_lse=True)
    assert luvc.check_status() == 0
    assert bool(out.isfinite().all())
    check(q, k, v, qs, ks, out, lse, bias=bias)
