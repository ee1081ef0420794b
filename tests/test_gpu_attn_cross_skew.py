"""Few tokens on the whole that are not evenly spread: most sequences have none, one has many, and its states are many too.  Which form computes such a
call follows from lengths that only the device knows.  The bounds are those of test_gpu_attn_cross."""
import math

import pytest
import torch

from test_gpu_attn_cross import check, inputs, ints, luvc, starts_of  # noqa: F401

pytestmark = pytest.mark.gpu

EVEN, SKEWED = ([1] * 64, [1000] * 64), ([0] * 20 + [60] + [0] * 42 + [4], [40] * 20 + [58000] + [30] * 42 + [1200])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,heads,D,queries,keys", [
    (4, 2, 64, [0] * 1023 + [1024], [3] * 1023 + [16384]), (4, 2, 64, [1000] + [0] * 1000 + [24], [9000] + [0] * 1000 + [9]),
    (16, 8, 128, [0, 0, 40, 0, 0, 3] + [0] * 40, [5, 900, 7001, 0, 0, 3000] + [300] * 40), (28, 4, 128, *EVEN), (28, 4, 128, *SKEWED),
    (3, 1, 256, [0] * 300 + [200] + [1] * 100, [20] * 300 + [5000] + [40] * 100)])
def test_few_tokens_of_one_sequence(luvc, dtype, hq, heads, D, queries, keys):  # noqa: F811
    q, k, v, qs, ks = inputs(dtype, hq, heads, D, queries, keys, seed=D, q_more=3, k_before=2, k_more=5)
    bias = torch.randn(k.shape[0], generator=torch.Generator().manual_seed(1)).cuda()
    bias[::5] = -math.inf
    for b in (None, bias):
        out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
        out, lse = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, key_bias=b, want_lse=True, out=out)
        assert luvc.check_status() == 0
        check(q, k, v, qs, ks, out, lse, bias=b)
        assert bool((out[-3:] == 7.0).all())
        assert torch.equal(luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, key_bias=b)[:-3], out[:-3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_captured_call_follows_its_lengths(luvc, dtype):  # noqa: F811
    """One graph, one workspace, even and skewed lengths in turn."""
    q, k, v, qs, ks = inputs(dtype, 28, 4, 128, EVEN[0], [1000] * 64, seed=2)
    skewed = starts_of(SKEWED[0]), starts_of(SKEWED[1])
    assert int(skewed[0][-1]) == q.shape[0] and int(skewed[1][-1]) <= k.shape[0]
    even = qs.clone(), ks.clone()
    ws = torch.zeros(luvc.attn_cross_workspace_bytes(), dtype=torch.uint8, device="cuda")
    out = torch.zeros(q.shape, dtype=q.dtype, device="cuda")
    luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, workspace=ws, out=out)
    one_each = luvc.attn_cross(q, k, v, k_starts=ks)
    assert torch.equal(out, one_each)                           # the same form as without q_starts
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, workspace=ws, out=out)
    for lengths in (skewed, even, skewed, skewed, even):
        qs.copy_(lengths[0])
        ks.copy_(lengths[1])
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert luvc.check_status() == 0
        if lengths is even:
            assert torch.equal(out, one_each)
        else:
            check(q, k, v, qs, ks, out, None)
        assert not ws[:2048].any()                              # counters are zero again


def test_a_list_that_tokens_alone_would_make_too_long(luvc):  # noqa: F811
    """1024 tokens of one sequence, 2048 heads, 16384 states: more than 2^31 tiles of 16 states for each token alone, 2^21 for blocks of tokens."""
    g = torch.Generator(device="cuda").manual_seed(0)
    heads, D, tokens, states = 2048, 8, 1024, 16384
    q = torch.randn((tokens, heads, D), generator=g, device="cuda", dtype=torch.bfloat16)
    k, v = (torch.randn((states, heads, D), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    qs, ks = starts_of([0] * 1023 + [tokens]), starts_of([0] * 1023 + [states])
    out = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks)
    assert luvc.check_status() == 0
    some = [0, 1, 700, 2047]
    check(q[:, some], k[:, some], v[:, some], qs[-2:], ks[-2:], out[:, some], None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("queries,keys", [([2048, 60], [0, 300]), ([60] + [300] * 8, [1296] + [0] * 8), ([700], [0]), ([33] + [9, 0] * 100 + [70], [40] + [0] * 201),
                                          ([20] * 147 + [500], [0] * 100 + [60] * 47 + [0]), ([10] * 320 + [90], [30, 0] * 160 + [0])])
def test_many_tokens_without_states(luvc, dtype, queries, keys):  # noqa: F811
    """Beside others that have some, or alone."""
    q, k, v, qs, ks = inputs(dtype, 6, 2, 64, queries, keys, seed=3, q_more=2, k_more=1)
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    out, lse = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, want_lse=True, out=out)
    assert luvc.check_status() == 0
    check(q, k, v, qs, ks, out, lse)
    assert bool((out[-2:] == 7.0).all())
