"""Attention of one new token over a cache with a scale for each 16 tokens of a head, against the formula in 64 bits.

The bound of an output element, worked out from the inputs before anything is run: scores are fp32 sums of D products (each
product and each of the at most D additions may lose 2^-23 of the largest partial sum; queries lose 2^-25 of their largest element
when they are brought to half precision; the key's scale is a factor more); a weight exp(score) is off by that times
its own size, in the numerator and in the denominator; a weight enters its product with the values off by 2^-14 of the largest of its 16
tokens' weights at most; sums over t tokens may lose 2^-23 per 16 tokens; a block of values whose scale is below 2^-60 of
another's is off by 2^-60 of that one's values; the result is rounded once to bf16."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def luvc():
    import paper_2512_09010_b200 as luvc
    assert torch.cuda.is_available()
    luvc.check_status()
    return luvc


def build(luvc, lengths, heads, D, page, layers=1, seed=0, spread=1.0, pages=None):
    """A cache whose sequences lie on scattered pages; what no sequence holds is NaN, its scales too.  spread: of the logarithm (base 2)
    of the values' scales."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    need = [-(-n // page) for n in lengths]
    pages = pages or sum(need) + 3
    shape = (layers, pages, heads, page, D)
    k = torch.randn(shape, generator=g, device="cuda") + 1.5 * torch.randn((layers, 1, heads, 1, D), generator=g, device="cuda")
    v = torch.randn(shape, generator=g, device="cuda")
    at = shape[:3] + (page // 16,)
    k_scale = 2.0 ** torch.randint(-8, -4, at, generator=g, device="cuda").float()
    v_scale = 2.0 ** (spread * torch.randn(at, generator=g, device="cuda")).round() / 64
    k = (k / k_scale.repeat_interleave(16, dim=3)[..., None]).clamp(-448, 448)
    v = (v * 64).clamp(-448, 448)
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    held = torch.zeros((pages, page), dtype=torch.bool)
    max_pages = max(need + [1]) + 1
    table, used = torch.full((len(lengths), max_pages), -1, dtype=torch.int32), 0
    for b, n in enumerate(lengths):
        mine = order[used:used + need[b]]
        used += need[b]
        table[b, :need[b]] = torch.tensor(mine, dtype=torch.int32)
        for j, p in enumerate(mine):
            held[p, :max(0, min(page, n - j * page))] = True
    gone = ~held.cuda()[None, :, None, :, None]
    empty = ~held.view(pages, -1, 16).any(2).cuda()[None, :, None]
    c = luvc.KvCache(k.masked_fill(gone, math.nan).to(E4M3), v.masked_fill(gone, math.nan).to(E4M3), len(lengths), max_pages,
                     k_scale=k_scale.masked_fill(empty, math.nan).contiguous(), v_scale=v_scale.masked_fill(empty, math.nan).contiguous())
    c.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
    c.table.copy_(table)
    return c


def rows(cache, slot, layer, n):
    out, pages = [], cache.table[slot, :-(-n // cache.page_size)].long()
    for pool, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        x = pool.float()[layer][pages].double() * scale[layer][pages].double().repeat_interleave(16, dim=2)[..., None]
        out.append(x.transpose(1, 2).reshape(-1, cache.heads, cache.head_dim)[:n])
    return out


def check(cache, q, got, lse, layer=0, seqs=None, scale=None, bias=None):
    n, hq, D = q.shape
    group = hq // cache.heads
    scale = scale or D ** -0.5
    for i in range(n):
        slot = i if seqs is None else seqs[i]
        t = int(cache.lengths[slot])
        if t == 0:
            assert not got[i].any() and (lse is None or bool((lse[i] == -math.inf).all()))
            continue
        k, v = rows(cache, slot, layer, t)
        k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
        qi = q[i].double()
        s = torch.einsum("hd,thd->ht", qi, k) * scale
        size = torch.einsum("hd,thd->ht", qi.abs(), k.abs()) * scale
        off = size * (D + 3) * 2.0 ** -23 + s.abs() * 2.0 ** -23 + scale * 2.0 ** -25 * qi.abs().amax(1)[:, None] * k.abs().sum(2).t()
        if bias is not None:
            w = min(t, bias.shape[1])
            b = torch.zeros(t, dtype=torch.float64, device="cuda")
            b[:w] = bias[i, :w].double()
            s = s + b
            off = off + torch.where(b.isfinite(), b.abs(), 0.0) * 2.0 ** -23
        keep = s > -math.inf
        s, v = torch.where(keep, s, -math.inf), torch.where(keep.t()[:, :, None], v, 0.0)
        if not keep.any():
            assert not got[i].any()
            continue
        top = s.amax(1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(1, keepdim=True)
        p = p / total
        want, spread = torch.einsum("ht,thd->hd", p, v), torch.einsum("ht,thd->hd", p, v.abs())
        near = torch.nn.functional.pad(p, (0, -t % 16)).view(hq, -1, 16).amax(2).repeat_interleave(16, dim=1)[:, :t]
        wrong = torch.where(keep, off, 0.0).amax(1, keepdim=True)
        rel = 2 * wrong + (t / 16 + D + 64) * 2.0 ** -23
        bound = spread * rel * 1.01 + torch.einsum("ht,thd->hd", near, v.abs()) * 2.0 ** -14 + v.abs().amax(0) * 2.0 ** -59
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
        diff = (got[i].double() - want).abs()
        assert bool((diff <= bound).all()), (i, t, float((diff / bound).max()))
        if lse is not None:
            ref = (top + total.log())[:, 0]
            assert bool(((lse[i].double() - ref).abs() <= wrong[:, 0] + (t / 16 + 64) * 2.0 ** -23 + ref.abs() * 2.0 ** -22).all())


def queries(n, hq, D):
    return torch.randn((n, hq, D), generator=torch.Generator().manual_seed(D + n)).bfloat16().cuda()


SHAPES = [(28, 4, 128, 16), (8, 8, 64, 32), (12, 1, 256, 64), (6, 3, 80, 16), (40, 2, 48, 16), (3, 1, 144, 16), (16, 16, 16, 48), (32, 2, 112, 128)]
LENGTHS = [[1], [0, 1, 15, 16, 17, 0], [31, 32, 33, 100, 2, 5, 64, 63], [700, 1, 0, 1297], [4100]]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda x: "x".join(map(str, x))[:20])
def test_ragged_sequences(luvc, shape, lengths):
    hq, heads, D, page = shape
    c = build(luvc, lengths, heads, D, page, seed=len(lengths) + D, spread=2.0)
    q = queries(len(lengths), hq, D)
    out, lse = luvc.attn_decode(q, c, want_lse=True)
    assert luvc.check_status() == 0
    check(c, q, out, lse)


@pytest.mark.parametrize("lengths", [[16451, 3, 9000, 1], [40000], [300] * 70])
def test_long_and_many(luvc, lengths):
    heads = 1 if len(lengths) == 1 else 4
    c = build(luvc, lengths, heads, 128, 64, seed=1)
    q = queries(len(lengths), 7 * heads, 128)
    out, lse = luvc.attn_decode(q, c, want_lse=True)
    assert luvc.check_status() == 0
    check(c, q, out, lse)
    assert torch.equal(luvc.attn_decode(q, c), out)                                # the same bits


def test_layers_slots_scale_and_biases(luvc):
    c = build(luvc, [50, 200, 0, 77], 2, 64, 16, layers=3, seed=4)
    q = queries(5, 8, 64)
    seqs = [3, 1, 1, 2, 0]
    bias = torch.randn((5, 120), generator=torch.Generator().manual_seed(1)).cuda()
    bias[0, 10:30], bias[1], bias[2, ::2], bias[4] = -math.inf, torch.finfo(torch.float32).min, -math.inf, -math.inf
    out, lse = luvc.attn_decode(q, c, layer=2, seqs=ints(seqs), scale=0.3, key_bias=bias, want_lse=True)
    assert luvc.check_status() == 0
    check(c, q, out, lse, layer=2, seqs=seqs, scale=0.3, bias=bias)
    assert not out[4].any() and bool((lse[4] == -math.inf).all())                 # 50 tokens, all masked


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_masked_blocks_may_hold_anything(luvc):
    c = build(luvc, [64, 100], 2, 64, 16, seed=6)
    q = queries(2, 8, 64)
    bias = torch.zeros((2, 100), device="cuda")
    bias[:, 16:32] = -math.inf
    bias[0, 40:43] = -math.inf
    want = luvc.attn_decode(q, c, key_bias=bias)
    page = c.table[0, 1]
    c.k[0, page], c.v[0, page] = math.nan, math.nan
    c.k_scale[0, page], c.v_scale[0, page] = math.nan, math.inf
    c.v[0, c.table[1, 1]] = -448.0
    c.k[0, c.table[0, 2], :, 8:11], c.v[0, c.table[0, 2], :, 8:11] = math.nan, math.nan
    assert torch.equal(luvc.attn_decode(q, c, key_bias=bias), want)
    assert luvc.check_status() == 0


@pytest.mark.parametrize("far", [8, 30, 60])
def test_scales_far_apart(luvc, far):
    """Blocks of values that differ by 2^far: the small ones alone count where the large ones have no weight, and the other way round."""
    heads, D = 2, 64
    c = build(luvc, [400], heads, D, 16, seed=far, spread=0.0)
    pages = c.table[0, :25].long()
    c.v_scale[0, pages[::3]] *= 2.0 ** -far
    c.v_scale[0, pages[5::7]] *= 2.0 ** (far // 2)
    c.v_scale[0, pages[9]] = 2.0 ** -60
    c.v[0, pages[9]] = 0.0
    q = queries(1, 8, D)
    bias = torch.zeros((1, 400), device="cuda")
    for low in (0.0, -30.0, -80.0):
        for which in (slice(0, None, 3), slice(5, None, 7)):
            bias.zero_()
            bias.view(1, 25, 16)[:, which] = low
            out, lse = luvc.attn_decode(q, c, key_bias=bias, want_lse=True)
            check(c, q, out, lse, bias=bias)
    assert luvc.check_status() == 0


def test_zero_values_and_a_key_above_all(luvc):
    c = build(luvc, [1000], 1, 128, 16, seed=2)
    first = c.table[0, 0]
    c.v[0, first], c.v_scale[0, first] = 0.0, 2.0 ** -60
    q = queries(1, 4, 128)
    bias = torch.zeros((1, 16), device="cuda")
    bias[0, 0] = 14.0
    out, lse = luvc.attn_decode(q, c, key_bias=bias, want_lse=True)
    check(c, q, out, lse, bias=bias)


def test_written_rows_are_attended_to(luvc):
    """Rows that the library wrote, step by step: values enhanced, scales grown, pages forked and pruned on the way."""
    g = torch.Generator(device="cuda").manual_seed(0)
    heads, D = 4, 128
    pool = torch.zeros((1, 40, heads, 16, D), device="cuda").to(E4M3)
    scale = torch.zeros((1, 40, heads, 1), device="cuda")
    c = luvc.KvCache(pool, pool.clone(), 4, 12, k_scale=scale, v_scale=scale.clone())
    kv = torch.randn((150, 2 * heads, D), generator=g, device="cuda").bfloat16()
    luvc.kv_reserve(c, ints([100, 50]))
    luvc.kv_write(c, kv[:, :heads], kv[:, heads:], starts=ints([0, 100, 150]), sizes=torch.arange(1, 151, dtype=torch.int32, device="cuda"))
    luvc.kv_compact(c, ints([3]), ints([90]), ints([list(range(0, 90, 2))]), seqs=ints([0]))
    luvc.kv_fork(c, ints([0, 1]), ints([2, 3]))
    for step in range(20):
        kv = torch.randn((3, 2 * heads, D), generator=g, device="cuda").bfloat16() * (1 + step)
        luvc.kv_reserve(c, ints([1, 1, 1]), seqs=ints([2, 1, 3]))
        luvc.kv_write(c, kv[:, :heads], kv[:, heads:], seqs=ints([2, 1, 3]))
    assert luvc.check_status() == 0
    q = queries(4, 28, D)
    out, lse = luvc.attn_decode(q, c, want_lse=True)
    check(c, q, out, lse)


def test_pages_that_are_none_read_as_zeros(luvc):
    c = build(luvc, [40], 1, 64, 16, seed=8)
    q = queries(1, 4, 64)
    want = luvc.attn_decode(q, c)
    page = int(c.table[0, 1])
    c.table[0, 1] = -1
    got = luvc.attn_decode(q, c)
    c.table[0, 1], c.k[0, page], c.v[0, page], c.k_scale[0, page], c.v_scale[0, page] = page, 0.0, 0.0, 1.0, 1.0
    assert torch.equal(luvc.attn_decode(q, c), got) and not torch.equal(got, want)
