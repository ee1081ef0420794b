"""Attention of one new token over the paged cache against the formula in 64 bits.

The bound of an output element, worked out from the inputs before anything is run: scores are fp32 sums of D products (each
product and each of the at most D additions may lose 2^-23 of the largest partial sum, and an 8-bit cache's queries lose
2^-25 of their largest element when they are brought to half precision); a weight exp(score) is off by that times
its own size, in the numerator and in the denominator; weights enter their product with the values with at least 16 bits;
sums over t tokens may lose 2^-23 per 16 tokens; the result is rounded once to its type."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}


@pytest.fixture(scope="module")
def luvc():
    import paper_2512_09010_b200 as luvc
    assert torch.cuda.is_available()
    luvc.check_status()
    return luvc


def build(luvc, dtype, lengths, heads, D, page, layers=1, seed=0, nan=True, spare=3):
    """A cache whose sequences lie on scattered pages; everything no sequence holds is NaN."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + spare
    k = torch.randn((layers, pages, heads, page, D), generator=g, device="cuda")
    v = torch.randn((layers, pages, heads, page, D), generator=g, device="cuda")
    k += 1.5 * torch.randn((layers, 1, heads, 1, D), generator=g, device="cuda")
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    held = torch.zeros((pages, page), dtype=torch.bool)
    max_pages = max(need + [1]) + 1
    table, at = torch.full((len(lengths), max_pages), -1, dtype=torch.int32), 0
    for b, n in enumerate(lengths):
        mine = order[at:at + need[b]]
        at += need[b]
        table[b, :need[b]] = torch.tensor(mine, dtype=torch.int32)
        for j, p in enumerate(mine):
            held[p, :max(0, min(page, n - j * page))] = True
    scales = {}
    if dtype == "e4m3":
        scales = {"k_scale": 0.01 + 0.02 * torch.rand((layers, heads), generator=g, device="cuda"),
                  "v_scale": 0.01 + 0.02 * torch.rand((layers, heads), generator=g, device="cuda")}
        k /= scales["k_scale"][:, None, :, None, None]
        v /= scales["v_scale"][:, None, :, None, None]
        k.clamp_(-448, 448), v.clamp_(-448, 448)
    if nan:
        gone = ~held.cuda()[None, :, None, :, None]
        k.masked_fill_(gone, math.nan), v.masked_fill_(gone, math.nan)
    c = luvc.KvCache(k.to(TYPES[dtype]), v.to(TYPES[dtype]), len(lengths), max_pages, **scales)
    c.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
    c.table.copy_(table)
    return c


def rows(cache, slot, layer, n):
    out = []
    for pool, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        pages = cache.table[slot, :-(-n // cache.page_size)].long()
        x = pool.float()[layer][pages].transpose(1, 2).reshape(-1, cache.heads, cache.head_dim)[:n].double()
        out.append(x if scale is None else x * scale[layer].double()[:, None])
    return out


def check(luvc, cache, q, got, lse, layer=0, seqs=None, scale=None, bias=None):
    n, hq, D = q.shape
    group = hq // cache.heads
    scale = scale or D ** -0.5
    u = 2.0 ** -24 if q.dtype == torch.float32 else 2.0 ** -8
    for i in range(n):
        slot = i if seqs is None else seqs[i]
        t = int(cache.lengths[slot])
        if t == 0:
            assert not got[i].any()
            assert lse is None or bool((lse[i] == -math.inf).all())
            continue
        k, v = rows(cache, slot, layer, t)
        k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
        qi = q[i].double()
        s = torch.einsum("hd,thd->ht", qi, k) * scale
        size = torch.einsum("hd,thd->ht", qi.abs(), k.abs()) * scale
        off = size * (D + 2) * 2.0 ** -23 + s.abs() * 2.0 ** -23
        if cache.dtype == torch.float8_e4m3fn:
            off = off + scale * 2.0 ** -25 * qi.abs().amax(1)[:, None] * k.abs().sum(2).t()
        if bias is not None:
            w = min(t, bias.shape[1])
            b = torch.zeros(t, dtype=torch.float64, device="cuda")
            b[:w] = bias[i, :w].double()
            s = s + b
            off = off + torch.where(b.isfinite(), b.abs(), 0.0) * 2.0 ** -23
        keep = s > -math.inf
        s, v = torch.where(keep, s, -math.inf), torch.where(keep.t()[:, :, None], v, 0.0)
        top = s.amax(1, keepdim=True)
        if not keep.any():
            assert not got[i].any()
            continue
        p = torch.exp(s - top)
        total = p.sum(1, keepdim=True)
        p = p / total
        want = torch.einsum("ht,thd->hd", p, v)
        spread = torch.einsum("ht,thd->hd", p, v.abs())
        wrong = torch.where(keep, off, 0.0).amax(1, keepdim=True)
        rel = 2 * wrong + 2 * 2.0 ** -17 * (q.dtype != torch.float32) + (t / 16 + D + 64) * 2.0 ** -23
        bound = spread * rel * 1.01 + u * want.abs()
        diff = (got[i].double() - want).abs()
        assert bool((diff <= bound).all()), (i, t, float((diff / bound).max()))
        if lse is not None:
            ref = (top + total.log())[:, 0]
            assert bool(((lse[i].double() - ref).abs() <= wrong[:, 0] + (t / 16 + 64) * 2.0 ** -23 + ref.abs() * 2.0 ** -22).all())


SHAPES = [  # type, query heads, key heads, D, page
    ("bf16", 28, 4, 128, 16), ("bf16", 32, 8, 128, 64), ("bf16", 8, 8, 64, 16), ("bf16", 16, 2, 80, 48), ("bf16", 24, 1, 256, 32),
    ("bf16", 17, 1, 8, 16), ("bf16", 10, 2, 104, 16), ("bf16", 32, 1, 192, 16), ("bf16", 66, 2, 64, 16),
    ("e4m3", 28, 4, 128, 16), ("e4m3", 8, 8, 64, 32), ("e4m3", 12, 1, 256, 64), ("e4m3", 6, 3, 80, 16), ("e4m3", 40, 2, 48, 16),
    ("e4m3", 3, 1, 144, 16),
    ("f32", 3, 1, 128, 16), ("f32", 12, 3, 256, 16), ("f32", 2, 2, 256, 32), ("f32", 5, 5, 100, 16), ("f32", 8, 2, 64, 64),
    ("f32", 16, 16, 64, 16), ("f32", 28, 4, 128, 48), ("f32", 4, 2, 20, 16), ("f32", 9, 1, 256, 16), ("f32", 34, 2, 68, 32),
]
LENGTHS = [[1], [0, 1, 15, 16, 17, 0], [31, 32, 33, 100, 2, 5, 64, 63], [700, 1, 0, 1297], [4100]]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda x: "x".join(map(str, x))[:20])
def test_ragged_sequences(luvc, shape, lengths):
    dtype, hq, heads, D, page = shape
    c = build(luvc, dtype, lengths, heads, D, page, seed=len(lengths) + D)
    q = torch.randn((len(lengths), hq, D), generator=torch.Generator().manual_seed(D)).to(c.io_dtype).cuda()
    out, lse = luvc.attn_decode(q, c, want_lse=True)
    assert luvc.check_status() == 0
    check(luvc, c, q, out, lse)


@pytest.mark.parametrize("dtype,heads,D", [("bf16", 8, 128), ("e4m3", 4, 128), ("f32", 2, 64), ("bf16", 1, 64), ("f32", 1, 256)])
def test_long_and_many(luvc, dtype, heads, D):
    lengths = [16451, 3, 9000, 1] if heads > 1 else [40000]
    c = build(luvc, dtype, lengths, heads, D, 64, seed=5, nan=True)
    q = torch.randn((len(lengths), 4 * heads, D), generator=torch.Generator().manual_seed(1)).to(c.io_dtype).cuda()
    check(luvc, c, q, *luvc.attn_decode(q, c, want_lse=True))
    lengths = [(37 * i) % 90 for i in range(600)]
    c = build(luvc, dtype, lengths, heads, D, 16, seed=6)
    q = torch.randn((600, 4 * heads, D), generator=torch.Generator().manual_seed(2)).to(c.io_dtype).cuda()
    check(luvc, c, q, *luvc.attn_decode(q, c, want_lse=True))


@pytest.mark.parametrize("dtype,q_heads,heads,D,tokens", [("bf16", 12, 1, 256, 30000), ("bf16", 32, 1, 128, 50000), ("e4m3", 8, 1, 128, 60000),
                                                          ("f32", 7, 1, 256, 9000), ("bf16", 2, 2, 8, 40000)])
def test_one_long_sequence_is_joined_across_all_ctas(luvc, dtype, q_heads, heads, D, tokens):
    c = build(luvc, dtype, [tokens], heads, D, 32, seed=D)
    q = torch.randn((1, q_heads, D), generator=torch.Generator().manual_seed(D)).to(c.io_dtype).cuda()
    out, lse = luvc.attn_decode(q, c, want_lse=True)
    check(luvc, c, q, out, lse)
    for _ in range(4):
        assert torch.equal(luvc.attn_decode(q, c), out)


@pytest.mark.parametrize("dtype,q_heads,heads,D", [("e4m3", 5, 5, 16), ("e4m3", 10, 2, 48), ("e4m3", 16, 1, 64), ("e4m3", 40, 2, 64), ("e4m3", 16, 16, 64),
                                                   ("f32", 12, 1, 256), ("f32", 18, 2, 200), ("f32", 5, 1, 132), ("f32", 14, 2, 112), ("f32", 20, 1, 128)])
def test_short_and_long_rows(luvc, dtype, q_heads, heads, D):
    for lengths, page in (([1, 0, 700, 63, 16, 17, 333], 48), ([3300], 16), ([95] * 40, 32)):
        c = build(luvc, dtype, lengths, heads, D, page, seed=q_heads + len(lengths), nan=True)
        q = torch.randn((len(lengths), q_heads, D), generator=torch.Generator().manual_seed(D)).to(c.io_dtype).cuda()
        check(luvc, c, q, *luvc.attn_decode(q, c, want_lse=True))
    bias = torch.randn((40, 80), generator=torch.Generator().manual_seed(4)).cuda()
    bias[3] = -float("inf")
    bias[5, 7:50] = torch.finfo(torch.float32).min
    check(luvc, c, q, *luvc.attn_decode(q, c, key_bias=bias, want_lse=True), bias=bias)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "f32"])
def test_biases_and_masks(luvc, dtype):
    lengths = [200, 33, 16, 70, 40]
    c = build(luvc, dtype, lengths, 2, 64, 16, seed=9)
    g = torch.Generator().manual_seed(3)
    q = torch.randn((5, 6, 64), generator=g).to(c.io_dtype).cuda()
    wide = torch.randn((5, 300), generator=g).cuda()
    bias = wide[:, :130]                                          # a part of a wider tensor; tokens from 130 on get 0
    check(luvc, c, q, *luvc.attn_decode(q, c, key_bias=bias, want_lse=True), bias=bias)
    bias = bias.clone()
    bias[0, ::3] = -math.inf
    bias[1, :] = -math.inf                                        # nothing is left: a row of zeros
    bias[2, 1:] = -math.inf
    bias[3, :] = torch.finfo(torch.float32).min                   # the lowest value everywhere: equal weights, not none
    bias[4, :39] = torch.finfo(torch.float32).min
    for page in c.table[0, :13].tolist():                         # rows under a mask may hold anything
        rowsel = [j for j in range(16) if (c.table[0].tolist().index(page) * 16 + j) % 3 == 0]
        for pool, what in ((c.k, math.nan), (c.v, math.inf if dtype != "e4m3" else math.nan)):
            flat = pool.float()
            flat[0, page, :, [j for j in rowsel if c.table[0].tolist().index(page) * 16 + j < 130]] = what
            pool.copy_(flat.to(pool.dtype))
    out, lse = luvc.attn_decode(q, c, key_bias=bias, want_lse=True)
    clean = build(luvc, dtype, lengths, 2, 64, 16, seed=9)
    check(luvc, clean, q, out, lse, bias=bias)
    assert not out[1].any() and bool((lse[1] == -math.inf).all())
    mean = rows(clean, 3, 0, 70)[1].mean(0).repeat_interleave(3, 0)
    assert ((out[3].double() - mean).abs() <= 2.0 ** -8 * mean.abs() + 1e-4).all()
    last = rows(clean, 4, 0, 40)[1][39].repeat_interleave(3, 0)   # the one token that is not masked
    assert ((out[4].double() - last).abs() <= 2.0 ** -8 * last.abs() + 1e-6).all()


@pytest.mark.parametrize("q_heads,heads,D", [(32, 8, 128), (5, 5, 64), (12, 1, 256), (28, 4, 80), (3, 1, 32)])
@pytest.mark.parametrize("gap", [6, 10, 14, 18, 30])
def test_small_weights_of_an_8_bit_cache(luvc, q_heads, heads, D, gap):
    """A token whose score is far above all others and whose value row is zero (for every other head): what is left are the small weights.

    They enter their product as the sum of two halves of 11 bits, in steps of 2^-24 of what 1 stands for; a rounding is off by 2^-25.
    The largest weight of 16 tokens is at least e^-6 there, and e^8 where the largest weight of all is among them.  A warp's part of
    the tokens begins anywhere, so every 16 tokens are given the larger bound of the tiles they can be in."""
    lengths = [700, 1, 16, 40, 333, 2500]
    c = build(luvc, "e4m3", lengths, heads, D, 16, seed=gap + D, nan=True)
    q = 0.3 * torch.randn((len(lengths), q_heads, D), generator=torch.Generator().manual_seed(D))
    q[:, :, 0] = 0.0
    q[:, ::2, 0] = 80.0
    q = q.bfloat16().cuda()
    c.k.view(torch.uint8)[..., 0] = 0
    for slot, t in enumerate([0, 0, 5, 39, 200, 1777]):
        page, at = int(c.table[slot, t // 16]), t % 16
        top = gap * D ** 0.5 / 80 / c.k_scale[0]
        assert float(top.max()) < 448
        c.k[0, page, :, at, 0] = top.to(torch.float8_e4m3fn)
        c.v.view(torch.uint8)[0, page, :, at] = 0
    out, lse = luvc.attn_decode(q, c, want_lse=True)
    assert luvc.check_status() == 0
    for i, n in enumerate(lengths):
        k, v = (x.repeat_interleave(q_heads // heads, 1) for x in rows(c, i, 0, n))
        s = torch.einsum("hd,thd->ht", q[i].double(), k) * D ** -0.5
        size = torch.einsum("hd,thd->ht", q[i].double().abs(), k.abs()) * D ** -0.5
        off = (size * (D + 3) * 2.0 ** -23 + D ** -0.5 * 2.0 ** -25 * q[i].double().abs().amax(1)[:, None] * k.abs().sum(2).t()).amax(1, keepdim=True)
        top = s.amax(1, keepdim=True)
        w = torch.exp(s - top)
        total = w.sum(1, keepdim=True)
        tiles = torch.nn.functional.pad(w, (0, -n % 16)).view(q_heads, -1, 16).amax(2)
        floor = torch.where(tiles == 1.0, math.exp(-8), tiles * math.exp(6)).repeat_interleave(16, 1)[:, :n] * 2.0 ** -25
        want = torch.einsum("ht,thd->hd", w / total, v)
        spread = torch.einsum("ht,thd->hd", w / total, v.abs())
        bound = (2.0 ** -8 * want.abs() + spread * (2 * off + 2 * 2.0 ** -17 + (n / 16 + D + 64) * 2.0 ** -23)
                 + torch.einsum("ht,thd->hd", floor / total, v.abs())) * 1.01
        diff = (out[i].double() - want).abs()
        assert bool((diff <= bound).all()), (i, n, float((diff / bound).max()))
        assert bool(((lse[i].double() - (top + total.log())[:, 0]).abs() <= off[:, 0] + (n / 16 + 64) * 2.0 ** -23 + top[:, 0].abs() * 2.0 ** -22).all())


def test_large_scores_and_a_scale(luvc):
    c = build(luvc, "bf16", [500, 77], 2, 128, 16, seed=11)
    q = 20 * torch.randn((2, 8, 128), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    check(luvc, c, q, *luvc.attn_decode(q, c, scale=0.5, want_lse=True), scale=0.5)
    big = build(luvc, "e4m3", [500, 77], 2, 128, 16, seed=11)
    q = (1e30 * torch.randn((2, 8, 128), generator=torch.Generator().manual_seed(4))).bfloat16().cuda()   # beyond half precision's range
    check(luvc, big, q, *luvc.attn_decode(q, big, scale=1e-31, want_lse=True), scale=1e-31)


def test_a_nan_in_a_row_that_counts_is_seen(luvc):
    c = build(luvc, "bf16", [100], 1, 64, 16, seed=12)
    q = torch.randn((1, 2, 64), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    c.k[0, int(c.table[0, 2]), 0, 5, 7] = math.nan
    assert bool(luvc.attn_decode(q, c).isnan().all())


@pytest.mark.parametrize("dtype,q_heads,heads,D", [("bf16", 28, 4, 128), ("bf16", 12, 1, 64), ("bf16", 6, 2, 200), ("f32", 28, 4, 128), ("f32", 16, 2, 60),
                                                   ("f32", 12, 1, 128), ("f32", 34, 2, 64), ("f32", 4, 4, 128), ("f32", 12, 1, 256)])
@pytest.mark.parametrize("what", ["v inf", "v both", "v nan", "v large", "k inf", "k -inf", "k nan", "k large", "q large"])
def test_what_is_not_finite_counts_as_the_formula_says(luvc, dtype, q_heads, heads, D, what):
    """Infinities, NaN (also the one arithmetic gives) and values near the ends of the range, in rows that count: an infinite value makes
    its column infinite and leaves the others; a score of -inf has weight zero; NaN goes through; large finite values stay finite."""
    lengths = [300, 2000]
    c = build(luvc, dtype, lengths, heads, D, 16, seed=D + q_heads, nan=False)
    q = torch.randn((2, q_heads, D), generator=torch.Generator().manual_seed(7)).to(c.io_dtype).cuda()
    nan = torch.tensor(0x7fffffff, dtype=torch.int32).view(torch.float32).item() if dtype == "f32" else math.nan

    def put(pool, slot, token, d, x):
        cell = pool[0, int(c.table[slot, token // 16]), :, token % 16, d]
        if dtype == "f32" and x != x:                             # the very bits
            cell.view(torch.int32).fill_(0x7fffffff if token % 2 else -1)
        else:
            cell.fill_(x)

    group = q_heads // heads
    for slot, tokens in enumerate(([5, 131], [44, 1700, 1999])):
        for t in tokens:
            if what == "v inf":
                put(c.v, slot, t, 3, math.inf), put(c.v, slot, t, D - 1, -math.inf)
            elif what == "v both":
                put(c.v, slot, t, 3, math.inf if t % 2 else -math.inf)
            elif what == "v nan":
                put(c.v, slot, t, 3, nan)
            elif what == "v large":
                put(c.v, slot, t, 3, 1e35), put(c.v, slot, t, 5, -1e35)
            elif what in ("k inf", "k -inf"):                     # "k -inf": the same sign for every head, so that all scores of t are -inf
                put(c.k, slot, t, 2, math.inf if what == "k inf" else -math.inf)
            elif what == "k nan":
                put(c.k, slot, t, 2, nan)
            elif what == "k large":
                put(c.k, slot, t, 2, 1e37)
    if what == "k -inf":
        q[:, :, 2] = q[:, :, 2].abs() + 0.25
    if what == "k large":
        q[:, :, 2] *= 1e-37
    if what == "q large":
        q[:, :, 2] *= 1e36
        c.k[..., 2] *= 1e-36
    out, lse = luvc.attn_decode(q, c, want_lse=True)
    assert luvc.check_status() == 0
    u = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
    for i, n in enumerate(lengths):
        k, v = (x.repeat_interleave(group, 1) for x in rows(c, i, 0, n))
        s = torch.einsum("hd,thd->ht", q[i].double(), k) * D ** -0.5
        p = torch.exp(s - s.amax(1, keepdim=True))
        p = p / p.sum(1, keepdim=True)
        term = p.t()[:, :, None] * v
        want = term.sum(0)
        size = (q[i].double()[:, None].abs() * k.transpose(0, 1).abs()).sum(2) * D ** -0.5
        off = torch.where(size.isfinite(), size, 0.0).amax(1, keepdim=True) * (D + 3) * 2.0 ** -23      # of scores, as above
        bound = term.abs().sum(0) * (2 * off + 2 * 2.0 ** -17 * (dtype != "f32") + (n / 16 + D + 64) * 2.0 ** -23) * 1.01 + u * want.abs()
        got = out[i].double()
        assert torch.equal(got.isnan(), want.isnan()), (i, int(got.isnan().sum()), int(want.isnan().sum()))
        assert torch.equal(got.isinf(), want.isinf()) and torch.equal(got[got.isinf()], want[want.isinf()])
        fine = want.isfinite()
        assert bool(((got - want).abs() <= bound)[fine].all())
        assert torch.equal(lse[i].isnan(), s.isnan().any(1) | (s == math.inf).any(1))
    assert what in ("k inf", "k nan") or bool(out.isfinite().any())


@pytest.mark.parametrize("dtype,q_heads,heads,D", [("e4m3", 4, 1, 64), ("e4m3", 12, 1, 128), ("bf16", 4, 1, 64), ("f32", 8, 1, 64), ("f32", 2, 1, 64)])
def test_masks_of_the_lowest_value_in_turn_with_tokens_that_count(luvc, dtype, q_heads, heads, D):
    """Every other 16 tokens carry the lowest bias, or one far below all others: the weights' reference does not follow them and back."""
    n = 200000
    c = build(luvc, dtype, [n, 333], heads, D, 16, seed=8, nan=False)
    c.v.view(torch.uint8).zero_()
    c.v.copy_((torch.ones(c.v.shape, device="cuda") * 1.75).to(c.v.dtype))            # equal values: the mean is exact but for the sums
    q = torch.randn((2, q_heads, D), generator=torch.Generator().manual_seed(1)).to(c.io_dtype).cuda()
    t = torch.arange(n, device="cuda") // 16 % 2
    for low in (torch.finfo(torch.float32).min, -200.0, -90.0):
        bias = torch.where(t == 1, low, 0.0).expand(2, n).contiguous()
        out, lse = luvc.attn_decode(q, c, key_bias=bias, want_lse=True)
        want = 1.75 * (c.v_scale[0] if c.v_scale is not None else torch.ones(1, device="cuda")).double()
        u = 2.0 ** -8 if dtype != "f32" else 2.0 ** -24
        # numerator and denominator are sums of the same weights: what is left is the rounding of 16-bit weights and of the sums
        rel = 2 * 2.0 ** -17 * (dtype != "f32") + (n / 16 / 148 + 64) * 2.0 ** -23
        assert bool(((out.double() - want).abs() <= (u + rel) * want).all()), (low, float((out.double() / want - 1).abs().max()))
        check(luvc, c, q[1:], out[1:], lse[1:], seqs=[1], bias=bias[1:])


@pytest.mark.parametrize("dtype,q_heads,heads,D", [("bf16", 28, 4, 128), ("bf16", 12, 1, 64), ("f32", 28, 4, 128), ("f32", 12, 1, 128), ("f32", 4, 4, 128),
                                                   ("f32", 8, 2, 64), ("f32", 12, 1, 256)])
def test_the_largest_values_do_not_overflow(luvc, dtype, q_heads, heads, D):
    # a weight is at most 1 relative to the largest, so the weighted sum stays finite where the formula's does; a warp reads many tokens
    # in turn, and one of them scores as much above those before it as their weights' reference may lag behind
    n, group = 60000, q_heads // heads
    c = build(luvc, dtype, [n], heads, D, 16, seed=D, nan=False)
    c.k.zero_()
    q = torch.ones((1, q_heads, D), dtype=c.io_dtype, device="cuda")
    big = 3.0e38
    for t, score, sign in ((3, 0.0, 1), (40, 5.5, 1), (45, 0.0, -1), (31000, 5.5, -1), (59999, 2.0, 1)):
        page = int(c.table[0, t // 16])
        c.k[0, page, :, t % 16, 0] = score * D ** 0.5
        c.v[0, page, :, t % 16, 3] = big * sign
    out = luvc.attn_decode(q, c)[0].double()
    k, v = (x.repeat_interleave(group, 1) for x in rows(c, 0, 0, n))
    s = torch.einsum("hd,thd->ht", q[0].double(), k) * D ** -0.5
    p = torch.softmax(s, 1)
    want, spread = torch.einsum("ht,thd->hd", p, v), torch.einsum("ht,thd->hd", p, v.abs())
    off = 5.5 * (D + 3) * 2.0 ** -23
    u = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
    bound = spread * (2 * off + 2 * 2.0 ** -17 * (dtype != "f32") + (n / 16 + D + 64) * 2.0 ** -23) * 1.01 + u * want.abs()
    assert bool((want.abs() < 3.0e38).all()) and bool(((out - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layers_slots_strides_and_streams(luvc, dtype):
    c = build(luvc, dtype, [100, 0, 45, 300], 2, 64, 16, layers=3, seed=13)
    g = torch.Generator().manual_seed(5)
    wide = torch.randn((5, 3 * 8 * 64), generator=g).to(c.io_dtype).cuda()
    q = wide[:, 8 * 64:16 * 64].view(5, 8, 64)                    # the middle part of a projection's rows
    seqs = torch.tensor([3, 0, 3, 1, 2], dtype=torch.int32, device="cuda")
    side, ws = torch.cuda.Stream(), torch.zeros(luvc.attn_workspace_bytes(), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        out, lse = luvc.attn_decode(q, c, layer=2, seqs=seqs, want_lse=True, workspace=ws)
    side.synchronize()
    check(luvc, c, q, out, lse, layer=2, seqs=seqs.tolist())
    again = torch.empty_like(out)
    for _ in range(3):                                            # the same bits every time
        assert torch.equal(luvc.attn_decode(q, c, layer=2, seqs=seqs, out=again, workspace=ws), out)
    bad = seqs.clone()
    bad[1] = 4                                                    # no such slot: empty, and reported
    got = luvc.attn_decode(q, c, layer=2, seqs=bad)
    assert luvc.check_status() == 2 and not got[1].any()
    rest = torch.tensor([0, 2, 3, 4], device="cuda")              # the others are right (the split of the work may differ)
    check(luvc, c, q[rest], got[rest], None, layer=2, seqs=seqs[rest].tolist())


@pytest.mark.parametrize("q_heads,heads,D", [(7, 1, 128), (16, 2, 80), (5, 1, 68), (12, 1, 128), (12, 1, 256), (18, 3, 100)])
def test_every_number_of_parts_around_a_full_ring(luvc, q_heads, heads, D):
    # Parts of one (sequence, head) that are joined at once fill shared memory up to the last one that fits (47 of 8 rows of 128
    # floats; 23 of 16).  One sequence of T tiles of 16 tokens has about T / 6 parts (six warps to a CTA, a tile for each), with
    # three or four warps more.
    for tokens in list(range(2100, 2500, 56)) + list(range(4300, 4760, 32)) + [4465, 4500, 4560]:
        c = build(luvc, "f32", [tokens], heads, D, 32, seed=tokens, nan=True)
        q = torch.randn((1, q_heads, D), generator=torch.Generator().manual_seed(D)).cuda()
        check(luvc, c, q, *luvc.attn_decode(q, c, want_lse=True))
    assert luvc.check_status() == 0


def test_results_repeat_bit_for_bit(luvc):
    c = build(luvc, "bf16", [9000, 100, 2500], 4, 128, 16, seed=14)
    q = torch.randn((3, 28, 128), generator=torch.Generator().manual_seed(6)).bfloat16().cuda()
    first = luvc.attn_decode(q, c)
    for _ in range(20):
        assert torch.equal(luvc.attn_decode(q, c), first)


@pytest.mark.parametrize("own", [False, True])
def test_calls_after_calls_that_overlapped_are_right(luvc, own):
    """Calls that share a workspace must not overlap, and what they give if they do is undefined; but when they have ended the workspace is
    as it was: calls that are kept in order from then on are right."""
    ws = torch.zeros(luvc.attn_workspace_bytes(), dtype=torch.uint8, device="cuda") if own else None
    g = torch.Generator().manual_seed(3)
    jobs = []
    shapes = (([30000], 8, 1, 64), ([2000], 8, 1, 64), ([5000, 700], 8, 2, 64), ([16451, 4173, 9000], 32, 8, 128), ([20000, 20001], 16, 4, 128),
              ([60000], 8, 2, 128), ([7000] * 7, 12, 3, 128))
    for i, (lengths, q_heads, heads, D) in enumerate(shapes):
        c = build(luvc, "bf16", lengths, heads, D, 16, seed=i, nan=False)
        q = torch.randn((len(lengths), q_heads, D), generator=g).bfloat16().cuda()
        jobs.append((c, q, luvc.attn_decode(q, c, workspace=ws)))
        check(luvc, c, q, jobs[-1][2], None)
    streams = [torch.cuda.Stream() for _ in range(4)]
    for a in range(len(jobs)):
        for b in range(len(jobs)):
            torch.cuda.synchronize()
            for k in range(12):
                for s, j in zip(streams, (a, b, b, a)):
                    with torch.cuda.stream(s):
                        luvc.attn_decode(jobs[j][1], jobs[j][0], workspace=ws)
            torch.cuda.synchronize()
            for c, q, want in jobs:
                for _ in range(2):
                    assert torch.equal(luvc.attn_decode(q, c, workspace=ws), want), (a, b)
    assert luvc.check_status() == 0


def test_reading_the_status_leaves_a_running_call_alone(luvc):
    """Another operator's wait gives up (made to, by the knobs of its status block), and the word is read while attention runs on another
    stream with the library's workspace."""
    c = build(luvc, "f32", [16451, 9000, 30000], 1, 256, 64, seed=2, nan=False)    # leaves room on the SMs for what else would run
    q = torch.randn((3, 12, 256), generator=torch.Generator().manual_seed(5)).cuda()
    want = luvc.attn_decode(q, c)
    x = torch.randn((3, 12, 12, 64), generator=torch.Generator().manual_seed(6)).cuda()
    luvc.oim_merge(x, 36)
    side, stream = torch.cuda.Stream(), torch.cuda.current_stream().cuda_stream
    outs = [torch.empty_like(want) for _ in range(12)]
    for _ in range(100):
        assert luvc.lib.luvc_debug_wait_probes(4, 1000, None, stream) == 0
        luvc.oim_merge(x, 36)                                     # gives up: the word is set
        assert luvc.lib.luvc_debug_wait_probes(0, 0, None, stream) == 0
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for o in outs:
                luvc.attn_decode(q, c, out=o)
        assert luvc.check_status() == 10
        torch.cuda.synchronize()
        assert luvc.check_status() == 0
        assert all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("dtype,q_heads,heads,D,lengths", [("bf16", 8, 1, 64, [40000]), ("bf16", 28, 4, 128, [97]), ("e4m3", 32, 8, 128, [3000, 20, 0, 900]),
                                                           ("f32", 16, 2, 64, [5000]), ("f32", 3, 1, 256, [2000, 2000]), ("f32", 28, 4, 128, [9, 3000])])
def test_a_wait_that_gives_up_is_reported_and_the_next_call_is_right(luvc, own, dtype, q_heads, heads, D, lengths):
    """The knobs of the status block let the first wait of the first warp run out, after a few thousand probes; nothing hangs.  The
    workspace is usable as it is afterwards."""
    c = build(luvc, dtype, lengths, heads, D, 16, seed=1, nan=False)
    q = torch.randn((len(lengths), q_heads, D), generator=torch.Generator().manual_seed(2)).to(c.io_dtype).cuda()
    stream = torch.cuda.current_stream().cuda_stream
    block = torch.zeros(4, dtype=torch.int32, device="cuda") if own else None
    options = dict(device_status=block, workspace=torch.zeros(luvc.attn_workspace_bytes(), dtype=torch.uint8, device="cuda")) if own else {}

    def read():
        return luvc.read_status(block) if own else luvc.check_status()

    want = luvc.attn_decode(q, c, **options)
    assert read() == 0
    check(luvc, c, q, want, None)
    for _ in range(3):
        assert luvc.lib.luvc_debug_wait_probes(5000, 1, block.data_ptr() if own else None, stream) == 0
        luvc.attn_decode(q, c, **options)
        torch.cuda.synchronize()
        assert luvc.lib.luvc_debug_wait_probes(0, 0, block.data_ptr() if own else None, stream) == 0
        assert torch.equal(luvc.attn_decode(q, c, **options), want)      # also while the word is set
        assert read() == 10 and read() == 0
        assert torch.equal(luvc.attn_decode(q, c, **options), want)
    if own:
        assert luvc.check_status() == 0
        assert not options["workspace"][:5 * 256 * 4].any()


def test_offsets_past_32_bits(luvc):
    # the last pages of a pool of more than 2^32 elements per tensor (8 GB of one byte each)
    heads, D, page = 8, 256, 64
    pages = (1 << 32) // (heads * D * page) + 40
    k = torch.zeros((1, pages, heads, page, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    v = torch.zeros((1, pages, heads, page, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    one = torch.ones((1, heads), device="cuda")
    c = luvc.KvCache(k, v, 2, 40, k_scale=one, v_scale=one)
    c.refs[:pages - 40].fill_(1)                                  # only the far end is free
    n = 30 * page + 5
    g = torch.Generator(device="cuda").manual_seed(8)
    new = torch.randn((2, n, heads, D), generator=g, device="cuda").bfloat16()
    count = torch.tensor([n], dtype=torch.int32, device="cuda")
    luvc.kv_reserve(c, count)
    assert c.table[0, :2].tolist() == [pages - 40, pages - 39]
    luvc.kv_write(c, new[0], new[1], starts=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    q = torch.randn((1, heads * 2, D), generator=g, device="cuda").bfloat16()
    k8, v8 = (x.float().to(torch.float8_e4m3fn).double() for x in new)
    s = torch.einsum("hd,thd->ht", q[0].double(), k8.repeat_interleave(2, 1)) / 16
    want = torch.einsum("ht,thd->hd", torch.softmax(s, 1), v8.repeat_interleave(2, 1))
    got = luvc.attn_decode(q, c)[0].double()
    assert luvc.check_status() == 0
    assert ((got - want).abs() <= 2.0 ** -8 * want.abs() + 2e-3).all()
    # dropping the first two thirds of its tokens moves rows within the far end
    idx = torch.arange(2 * n // 3, n, dtype=torch.int32, device="cuda")[None, :8 * page]
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    luvc.kv_compact(c, zero, count, idx.contiguous())
    assert luvc.check_status() == 0 and c.lengths[0] == 8 * page and int(c.table[0, 0]) >= pages - 9
    moved = c.k[0][c.table[0, :8].long().tolist()[0]].float().transpose(0, 1)
    assert torch.equal(moved, k8[2 * n // 3:2 * n // 3 + page].float())


def test_the_longest_sequence_of_an_8_bit_cache(luvc):
    # 2^31 - 20 tokens of one key head of 16 (32 GB of keys, 32 GB of values): the last 32-token tile ends past 2^31 - 1
    pages, page, D, n = (1 << 27) - 1, 16, 16, (1 << 31) - 20
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB")
    k = torch.zeros((1, pages, 1, page, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    v = torch.zeros((1, pages, 1, page, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    one = torch.ones((1, 1), device="cuda")
    c = luvc.KvCache(k, v, 1, pages, k_scale=one, v_scale=one)
    c.table.copy_(torch.arange(pages, dtype=torch.int32, device="cuda")[None])
    c.lengths.fill_(n)
    g = torch.Generator(device="cuda").manual_seed(1)
    live = n - (pages - 1) * page                                 # tokens of the last page; what follows them is NaN
    k.view(torch.uint8)[0, -1, 0, live:] = 0x7f
    v.view(torch.uint8)[0, -1, 0, live:] = 0x7f
    last = torch.randn((live, D), generator=g, device="cuda").to(torch.float8_e4m3fn)
    v[0, -1, 0, :live] = last
    k[0, -1, 0, :live, 0] = torch.full((live,), 8.0, device="cuda").to(torch.float8_e4m3fn)
    q = torch.zeros((1, 10, D), dtype=torch.bfloat16, device="cuda")
    q[0, :, 0] = torch.arange(10, device="cuda") + 8.0
    out, lse = luvc.attn_decode(q, c, scale=0.5, want_lse=True)   # the last tokens' scores are 4 (8 .. 17) = 32 .. 68, all others' 0
    assert luvc.check_status() == 0
    top = 4 * q[0, :, :1].double()
    total = live + (n - live) * torch.exp(-top)
    want = last.double().sum(0) / total
    # the weights of 4 equal keys and of the rest, summed in 32 bits in pieces of some 10^4 tiles (see check)
    rel = 2 * 2.0 ** -17 + 2 * 68 * 18 * 2.0 ** -23 + (n / 16 / 148 / 16 + 200) * 2.0 ** -23 * (1 - live / total)
    bound = 2.0 ** -8 * want.abs() + last.double().abs().sum(0) / total * (rel + 64 * 2.0 ** -23)
    assert bool(((out[0].double() - want).abs() <= bound).all())
    assert bool(((lse[0].double() - top[:, 0] - total[:, 0].log()).abs() <= rel[:, 0] + 68 * 2.0 ** -20).all())
    del c, k, v
    torch.cuda.empty_cache()
