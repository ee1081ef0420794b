"""Attention over a cache with a scale for each 16 tokens of a head, where a warp has several tiles of a part and scores and scales are far
apart within them: sums of weights, and the units of the sums of values, both move, and their product has to stay in range.  The bounds are those
of test_gpu_attn_block."""
import pytest
import torch

from test_gpu_attn_block import build, check, ints, luvc, queries  # noqa: F401

pytestmark = pytest.mark.gpu


def pattern(luvc, length, heads, D, exponent, seed):  # noqa: F811
    """Blocks in turn: values of 224 to 448 times 2^exponent; zeros, with the scale the library writes for them; values of about one."""
    c = build(luvc, [length], heads, D, 16, seed=seed, spread=0.0)
    pages = c.table[0, :-(-length // 16)].long()
    large, zero = pages[0::3], pages[1::3]
    g = torch.Generator(device="cuda").manual_seed(seed)
    shape = (large.numel(), heads, 16, D)
    c.v.view(torch.uint8)[0, large] = (224 + 224 * torch.rand(shape, generator=g, device="cuda")).to(c.v.dtype).view(torch.uint8)
    c.v_scale[0, large] = 2.0 ** exponent
    c.v.view(torch.uint8)[0, zero] = 0
    c.v_scale[0, zero] = 2.0 ** -60
    return c


@pytest.mark.parametrize("exponent", [-3, 0, 60])
@pytest.mark.parametrize("gap", [30.0, 34.0, 41.0, 50.0, 62.0, 68.0, 80.0])
def test_large_values_then_zeros_far_below(luvc, gap, exponent):  # noqa: F811
    length, heads, D = 30011, 8, 128                            # six or seven tiles for each warp
    c = pattern(luvc, length, heads, D, exponent, seed=int(gap))
    q = queries(1, 8, D)
    bias = torch.zeros((1, -(-length // 16), 16), device="cuda")
    bias[0, 0::3], bias[0, 2::3] = gap, gap - 10.0
    bias = bias.view(1, -1)[:, :length].contiguous()
    out, lse = luvc.attn_decode(q, c, scale=0.02, key_bias=bias, want_lse=True)
    assert luvc.check_status() == 0
    assert bool(out.isfinite().all())
    check(c, q, out, lse, scale=0.02, bias=bias)
    assert torch.equal(luvc.attn_decode(q, c, scale=0.02, key_bias=bias), out)


def test_zeros_far_below_without_biases(luvc):  # noqa: F811
    """The same from the keys: one direction that all queries share, long for the large values, missing for the zeros; scores 60, 50 and 0."""
    length, heads, D = 30011, 8, 64
    c = pattern(luvc, length, heads, D, -1, seed=3)
    pages = c.table[0, :-(-length // 16)].long()
    c.k.view(torch.uint8)[0, pages] = 0
    for at, stored in ((0, 60.0), (2, 52.0)):
        row = torch.zeros((pages[at::3].numel(), heads, 16, D), device="cuda")
        row[..., 5] = stored
        c.k.view(torch.uint8)[0, pages[at::3]] = row.to(c.k.dtype).view(torch.uint8)
    c.k_scale[0, pages] = 1.0
    q = torch.zeros((1, 8, D), dtype=torch.bfloat16, device="cuda")
    q[..., 5] = 1.0
    out, lse = luvc.attn_decode(q, c, scale=1.0, want_lse=True)
    assert luvc.check_status() == 0
    assert bool(out.isfinite().all())
    check(c, q, out, lse, scale=1.0)


@pytest.mark.parametrize("scale", [2.0 ** 127, 2.0 ** 100, 2.0 ** 60, 2.0 ** -60, 2.0 ** -126, 0.0, -1.0])
@pytest.mark.parametrize("lengths", [[30011], [100, 40]])
def test_scales_of_masked_blocks_count_for_nothing(luvc, lengths, scale):  # noqa: F811
    """Not for the precision of the others either: the same bits, whatever a masked block's scales are."""
    c = build(luvc, lengths, 4, 128, 16, seed=12)
    q = queries(len(lengths), 28, 128)
    bias = torch.zeros((len(lengths), -(-max(lengths) // 16), 16), device="cuda")
    bias[:, 1::3] = -float("inf")
    bias = bias.view(len(lengths), -1)[:, :max(lengths)].contiguous()
    want = luvc.attn_decode(q, c, key_bias=bias)
    check(c, q, want, None, bias=bias)
    for i, n in enumerate(lengths):
        masked = c.table[i, 1:-(-n // 16):3].long()
        c.k_scale[0, masked], c.v_scale[0, masked] = scale, scale
    assert torch.equal(luvc.attn_decode(q, c, key_bias=bias), want)
    assert luvc.check_status() == 0
