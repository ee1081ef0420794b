"""The paged cache in 8 bits with a scale for each 16 tokens of a head, against a plain model of its rows and scales: stored values and
scales have to be the model's, bit for bit, and so have the rows that are read back (products with powers of two, rounded once).
Only values that were enhanced by log(size) are compared with a bound: half a step of e4m3, 2^-4 of the value, or of its
smallest steps, 2^-10 of the scale, and 2^-22 of the sum for the logarithm."""
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


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def to_e4m3(x):
    """32-bit values to the nearest e4m3, saturated, NaN kept; as 32-bit values."""
    return x.clamp(-448, 448).to(E4M3).float()


def fitting(x):
    """[heads, rows, D]: for each head the smallest power of two from 2^-60 to 2^60 whose 448-fold no finite element exceeds."""
    top = torch.where(x.isfinite(), x.abs(), 0.0).double().amax((1, 2))
    e = torch.full_like(top, -60.0)
    for power in range(-60, 60):
        e = torch.where(top > 448.0 * 2.0 ** power, power + 1.0, e)
    return (2.0 ** e).float()


class Sequence:
    """Stored values [heads, tokens, D] and scales [heads, blocks] of the keys or the values of a sequence in one layer."""

    def __init__(self, heads, D):
        self.x, self.s = torch.zeros((heads, 0, D), device="cuda"), torch.zeros((heads, 0), device="cuda")

    def write(self, rows):                                   # [tokens, heads, D], 32 bits
        rows = rows.transpose(0, 1)
        old = self.x.shape[1]
        self.x = torch.cat((self.x, torch.zeros_like(rows)), dim=1)
        for b in range(old // 16, -(-self.x.shape[1] // 16) if rows.shape[1] else 0):
            lo, hi = max(old, 16 * b), min(self.x.shape[1], 16 * b + 16)
            new = rows[:, lo - old:hi - old]
            s = fitting(new)
            if 16 * b < old:
                was = self.s[:, b].clone()
                s = torch.maximum(s, was)
                self.x[:, 16 * b:old] = to_e4m3(self.x[:, 16 * b:old] * (was / s)[:, None, None])
                self.s[:, b] = s
            else:
                self.s = torch.cat((self.s, s[:, None]), dim=1)
            self.x[:, lo:hi] = to_e4m3(new / s[:, None, None])

    def keep(self, order, page):
        still = 0
        while (still + 1) * page <= len(order) and order[(still + 1) * page - 1] == (still + 1) * page - 1:
            still += 1
        pick = torch.tensor(order, dtype=torch.long, device="cuda")
        had, x = self.s[:, pick // 16], self.x[:, pick]
        now = torch.stack([had[:, b:b + 16].amax(1) for b in range(0, len(order), 16)], dim=1) if order else self.s[:, :0]
        now[:, :still * page // 16] = self.s[:, :still * page // 16]
        self.x = to_e4m3(x * (had / now.repeat_interleave(16, dim=1)[:, :len(order)])[..., None])
        self.s = now

    def copy(self):
        y = Sequence(self.x.shape[0], self.x.shape[2])
        y.x, y.s = self.x.clone(), self.s.clone()
        return y

    def rows(self):
        return (self.x * self.s.repeat_interleave(16, dim=1)[:, :self.x.shape[1], None]).transpose(0, 1)


class Rig:
    def __init__(self, luvc, heads, D, page, slots, tokens, layers=1, pages=None):
        self.luvc, self.heads, self.D, self.page, self.layers = luvc, heads, D, page, layers
        cols = -(-tokens // page) + 1
        pages = pages or slots * cols
        pool = torch.full((layers, pages, heads, page, D), float("nan"), device="cuda").to(E4M3)
        scale = torch.full((layers, pages, heads, page // 16), float("nan"), device="cuda")
        self.cache = luvc.KvCache(pool, pool.clone(), slots, cols, k_scale=scale, v_scale=scale.clone())
        self.model = [[[Sequence(heads, D) for _ in range(2)] for _ in range(layers)] for _ in range(slots)]

    def append(self, slots, parts, sizes=None):
        """parts: for each slot (k, v) of 16-bit rows [layers, tokens, heads, D]."""
        counts = [p[0].shape[1] for p in parts]
        starts = ints([sum(counts[:i]) for i in range(len(counts) + 1)])
        self.luvc.kv_reserve(self.cache, ints(counts), seqs=ints(slots))
        for layer in range(self.layers):
            both = torch.cat([torch.cat((k[layer], v[layer]), dim=1) for k, v in parts]) if sum(counts) else torch.zeros((0, 2 * self.heads, self.D)).bfloat16().cuda()
            self.luvc.kv_write(self.cache, both[:, :self.heads], both[:, self.heads:], layer=layer, starts=starts, seqs=ints(slots),
                               sizes=torch.cat(sizes) if sizes else None)
            for i, slot in enumerate(slots):
                k, v = parts[i][0][layer].float(), parts[i][1][layer].float()
                if sizes:
                    v = v + sizes[i].float().log()[:, None, None]
                self.model[slot][layer][0].write(k)
                self.model[slot][layer][1].write(v)

    def stored(self, slot, layer):
        n = int(self.cache.lengths[slot])
        at = self.cache.table[slot, :-(-n // self.page)].long()
        out = []
        for pool, scale in ((self.cache.k, self.cache.k_scale), (self.cache.v, self.cache.v_scale)):
            x = pool.float()[layer][at].transpose(0, 1).reshape(self.heads, -1, self.D)[:, :n]
            out.append((x, scale[layer][at].transpose(0, 1).reshape(self.heads, -1)[:, :-(-n // 16)]))
        return out

    def check(self, exact_values=True):
        assert self.luvc.check_status() == 0
        for slot, layers in enumerate(self.model):
            for layer, want in enumerate(layers):
                assert int(self.cache.lengths[slot]) == want[0].x.shape[1]
                for kind, (x, s) in enumerate(self.stored(slot, layer)):
                    assert torch.equal(s, want[kind].s), (slot, layer, kind)
                    if exact_values or kind == 0:
                        assert torch.equal(x.nan_to_num(1e9), want[kind].x.nan_to_num(1e9)), (slot, layer, kind)


def rows(g, layers, tokens, heads, D, size=1.0):
    x = torch.randn((2, layers, tokens, heads, D), generator=g, device="cuda") * size
    x = x * torch.exp(2 * torch.randn((2, layers, tokens, 1, 1), generator=g, device="cuda"))
    return x.bfloat16()[0], x.bfloat16()[1]


@pytest.mark.parametrize("heads,D,page", [(1, 16, 16), (4, 128, 16), (8, 128, 64), (3, 80, 48), (2, 256, 32), (5, 64, 128), (1, 208, 16), (17, 32, 16)])
def test_prompts_and_steps(luvc, heads, D, page):
    g = torch.Generator(device="cuda").manual_seed(D + heads)
    r = Rig(luvc, heads, D, page, 5, 400, layers=2)
    r.append([3, 0, 4], [rows(g, 2, n, heads, D) for n in (97, 1, 16)])
    r.check()
    r.append([1, 3, 0], [rows(g, 2, n, heads, D) for n in (0, 160, 31)])
    r.check()
    for step in range(19):                                   # a token each; ever larger ones bring blocks to new scales
        r.append([4, 0, 3, 1], [rows(g, 2, 1, heads, D, size=1.5 ** step) for _ in range(4)])
    r.check()


def test_many_tokens(luvc):
    g = torch.Generator(device="cuda").manual_seed(9)
    r = Rig(luvc, 2, 64, 32, 40, 3001)
    r.append(list(range(40)), [rows(g, 1, 1 + (i * 37) % 90, 2, 64) for i in range(40)])
    r.append([0, 1], [rows(g, 1, n, 2, 64) for n in (2901, 2000)])
    r.check()


@pytest.mark.parametrize("heads,D", [(4, 128), (3, 48)])
def test_enhanced_values(luvc, heads, D):
    g = torch.Generator(device="cuda").manual_seed(D)
    r = Rig(luvc, heads, D, 16, 3, 200)
    parts = [rows(g, 1, n, heads, D) for n in (33, 100, 7)]
    sizes = [torch.randint(1, 4000, (k.shape[1],), generator=g, device="cuda", dtype=torch.int32) for k, _ in parts]
    r.append([0, 1, 2], parts, sizes)
    r.check(exact_values=False)
    for slot in range(3):
        x, s = r.stored(slot, 0)[1]
        s = s.double().repeat_interleave(16, dim=1)[:, :x.shape[1], None]
        want = parts[slot][1][0].double().transpose(0, 1) + sizes[slot].double().log()[None, :, None]
        bound = torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * s) + 2.0 ** -22 * (want.abs() + 9)
        assert bool(((x.double() * s - want).abs() <= bound).all())


def test_extreme_rows(luvc):
    """Zeros, the smallest and largest numbers, infinities and NaN, alone and beside ordinary rows."""
    g = torch.Generator(device="cuda").manual_seed(3)
    heads, D = 2, 64
    r = Rig(luvc, heads, D, 16, 8, 64)
    parts = []
    for i in range(8):
        k, v = rows(g, 1, 21, heads, D)
        if i == 0:
            k.zero_()
        if i == 1:
            k[:, 3], v[:, 4, 0, 5] = math.inf, -math.inf
        if i == 2:
            k[:, 5, 1, 7], v[:, 20] = math.nan, math.nan
        if i == 3:
            k *= 2.0 ** -100
            v *= 2.0 ** 100
        if i == 4:
            k[:, :, :, ::2], v[:, 0] = 0.0, 3.3e38
        if i == 5:
            v[:, :16] *= 2.0 ** -80
            v[:, 16:] *= 2.0 ** 66
        if i == 6:
            k[:, :, 0], v[:, :, 1] = 1.75 * 2.0 ** 5, 1.765625 * 2.0 ** 5       # at the border of a scale, and past it
        parts.append((k, v))
    r.append(list(range(8)), parts)
    r.check()
    more = [rows(g, 1, 6, heads, D, size=2.0 ** (4 * i - 14)) for i in range(8)]
    r.append(list(range(8)), more)
    r.check()


@pytest.mark.parametrize("heads,D,page,layers", [(4, 128, 16, 2), (8, 64, 64, 1), (3, 80, 48, 3), (1, 256, 32, 1), (2, 16, 16, 1)])
def test_forked_pruned_and_grown(luvc, heads, D, page, layers):
    g = torch.Generator(device="cuda").manual_seed(page + D)
    r = Rig(luvc, heads, D, page, 9, 500, layers=layers)
    parts = [rows(g, layers, n, heads, D) for n in (301, 64, 17, 5)]
    r.append([0, 1, 2, 3], parts)
    r.luvc.kv_fork(r.cache, ints([0, 0, 2, 1]), ints([4, 5, 6, 7]))
    for src, dst in ((0, 4), (0, 5), (2, 6), (1, 7)):
        r.model[dst] = [[x.copy() for x in pair] for pair in r.model[src]]
    r.check()
    cuts = {0: (9, 280, sorted(torch.randperm(280, generator=torch.Generator().manual_seed(1))[:70].tolist())),
            5: (32, 200, list(range(0, 200, 3))), 2: (0, 17, []), 3: (1, 3, [0, 1, 2]), 7: (0, 64, list(range(40)) + [63])}
    keep = max(len(c[2]) for c in cuts.values())
    idx = torch.zeros((len(cuts), keep), dtype=torch.int32)
    for i, c in enumerate(cuts.values()):
        idx[i, :len(c[2])] = torch.tensor(c[2], dtype=torch.int32)
    r.luvc.kv_compact(r.cache, ints([c[0] for c in cuts.values()]), ints([c[1] for c in cuts.values()]), idx.cuda(),
                      counts=ints([len(c[2]) for c in cuts.values()]), seqs=ints(list(cuts)))
    for slot, (first, span, kept) in cuts.items():
        n = r.model[slot][0][0].x.shape[1]
        order = list(range(first)) + [first + j for j in kept] + list(range(first + span, n))
        for pair in r.model[slot]:
            for x in pair:
                x.keep(order, page)
    r.check()
    for step in range(18):
        slots = [0, 2, 3, 4, 5, 6, 7]
        r.append(slots, [rows(g, layers, 1, heads, D, size=3.0 * (step + 1)) for _ in slots])
    r.check()
    r.luvc.kv_free(r.cache, ints([1, 4]))
    for slot in (1, 4):
        r.model[slot] = [[Sequence(heads, D) for _ in range(2)] for _ in range(layers)]
    r.append([1, 8], [rows(g, layers, n, heads, D, size=1e-3) for n in (20, 50)])      # pages that others had: their scales are not kept
    r.check()


# ---- rows back ------------------------------------------------------------------------------------------------


def read(r, starts, tokens, spare=0, **how):
    both = torch.full((tokens + spare, 2 * r.heads, r.D), 7.0, dtype=r.cache.io_dtype, device="cuda")
    k, v = both[:, :r.heads], both[:, r.heads:]
    r.luvc.kv_read(r.cache, k, v, starts=ints(starts) if starts is not None else None, **how)
    return k, v


@pytest.mark.parametrize("heads,D,page", [(4, 128, 16), (3, 80, 48), (1, 256, 64), (6, 16, 16)])
def test_rows_back(luvc, heads, D, page):
    g = torch.Generator(device="cuda").manual_seed(heads)
    r = Rig(luvc, heads, D, page, 4, 900, layers=2)
    lengths = [130, 0, 871, 3]
    r.append([0, 1, 2, 3], [rows(g, 2, n, heads, D) for n in lengths])
    for layer in range(2):
        want = [torch.cat([r.model[s][layer][x].rows().bfloat16() for s in range(4)]) for x in range(2)]
        starts = [0, 130, 130, 1001, 1004]
        got = read(r, starts, 1004, spare=5, layer=layer)
        for x in range(2):
            assert torch.equal(got[x][:1004], want[x])
            assert bool((got[x][1004:] == 7.0).all())                               # behind the last sequence
        # parts, in another order, one of them twice
        got = read(r, [0, 10, 40, 41, 141], 141, layer=layer, seqs=ints([2, 0, 3, 2]), first=ints([861, 100, 2, 0]))
        pick = torch.tensor(list(range(130 + 861, 130 + 871)) + list(range(100, 130)) + [130 + 871 + 2] + list(range(130, 230)), device="cuda")
        for x in range(2):
            assert torch.equal(got[x], want[x][pick])
        got = read(r, None, 3, layer=layer, seqs=ints([3, 0, 3]), first=ints([1, 129, 0]))
        for x in range(2):
            assert torch.equal(got[x], want[x][torch.tensor([1002, 129, 1001], device="cuda")])
    assert luvc.check_status() == 0


def test_rows_that_are_not_there_are_zeros(luvc):
    g = torch.Generator(device="cuda").manual_seed(2)
    r = Rig(luvc, 2, 32, 16, 2, 40)
    r.append([0, 1], [rows(g, 1, n, 2, 32) for n in (20, 0)])
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    want = r.model[0][0][0].rows().bfloat16()
    k, _ = read(r, [0, 4, 6, 7, 8], 8, seqs=ints([0, 1, 5, -1]), first=ints([18, 0, 0, 0]), device_status=status)
    assert torch.equal(k[:2], want[18:]) and not k[2:].any()
    assert luvc.read_status(status) == 2
    k, _ = read(r, None, 1, first=ints([-1]), device_status=status)
    assert not k.any() and luvc.read_status(status) == 2
    k, _ = read(r, None, 1, first=ints([2147483647]), device_status=status)
    assert not k.any() and luvc.read_status(status) == 2
    r.cache.table[0, 1] = -1                                                        # a page that is none
    k, _ = read(r, [0, 20], 20, device_status=status)
    assert torch.equal(k[:16], want[:16]) and not k[16:].any() and luvc.read_status(status) == 2
    assert luvc.check_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32", "e4m3"])
def test_rows_back_from_the_other_caches(luvc, dtype):
    t = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": E4M3}[dtype]
    g = torch.Generator(device="cuda").manual_seed(5)
    pool = torch.randn((2, 9, 3, 16, 48), generator=g, device="cuda")
    scale = torch.rand((2, 3), generator=g, device="cuda") + 0.5 if dtype == "e4m3" else None
    c = luvc.KvCache(pool.to(t), pool.flip(0).contiguous().to(t), 2, 5, k_scale=scale, v_scale=scale)
    luvc.kv_reserve(c, ints([70, 33]))
    k = torch.empty((103, 3, 48), dtype=c.io_dtype, device="cuda")
    v = torch.empty_like(k)
    luvc.kv_read(c, k, v, layer=1, starts=ints([0, 70, 103]))
    assert luvc.check_status() == 0
    for got, p in ((k, c.k), (v, c.v)):
        x = p.float()[1] * (1.0 if scale is None else scale[1][:, None, None])
        flat = [x[c.table[s, :-(-n // 16)].long()].transpose(1, 2).reshape(-1, 3, 48)[:n] for s, n in ((0, 70), (1, 33))]
        assert torch.equal(got, torch.cat(flat).to(c.io_dtype))


def test_write_reports_rows_it_cannot_place(luvc):
    g = torch.Generator(device="cuda").manual_seed(6)
    r = Rig(luvc, 2, 32, 16, 2, 40)
    r.append([0, 1], [rows(g, 1, n, 2, 32) for n in (20, 3)])
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    k, v = rows(g, 1, 25, 2, 32)
    luvc.kv_write(r.cache, k[0], v[0], starts=ints([0, 25]), device_status=status)         # five more than the sequence has
    assert luvc.read_status(status) == 2
    for x, rows_ in ((0, k), (1, v)):
        s = Sequence(2, 32)
        s.write(rows_[0, 5:].float())
        got = r.stored(0, 0)[x]
        assert torch.equal(got[0], s.x) and torch.equal(got[1], s.s)
    luvc.kv_write(r.cache, k[0, :2], v[0, :2], seqs=ints([7, 1]), device_status=status)
    assert luvc.read_status(status) == 2
    r.model[1][0][0].x, r.model[1][0][1].x = r.model[1][0][0].x[:, :2], r.model[1][0][1].x[:, :2]
    r.model[1][0][0].write(k[0, 1:2].float()), r.model[1][0][1].write(v[0, 1:2].float())
    for x in range(2):
        got = r.stored(1, 0)[x]
        assert torch.equal(got[0], r.model[1][0][x].x) and torch.equal(got[1], r.model[1][0][x].s)
    assert luvc.check_status() == 0


@pytest.mark.parametrize("given", [1, 15, 16, 24, 33, 39])
def test_starts_past_the_rows_write_the_rows_there_are(luvc, given):
    """starts names 40 rows, the call has fewer: those are written, and no scale, stored row or read depends on what lies behind them."""
    r = Rig(luvc, 3, 64, 32, 1, 64)
    k, v = rows(torch.Generator("cuda").manual_seed(given), 1, 64, 3, 64)
    k[0, given:] = v[0, given:] = 1e6                        # behind the rows of the call, in the same memory
    luvc.kv_reserve(r.cache, ints([40]), seqs=ints([0]))
    table = r.cache.table[0].tolist()
    luvc.kv_write(r.cache, k[0, :given], v[0, :given], starts=ints([0, 40]), seqs=ints([0]))
    luvc.check_status()
    for pool, scale, x in ((r.cache.k, r.cache.k_scale, k), (r.cache.v, r.cache.v_scale, v)):
        model = Sequence(3, 64)
        model.write(x[0, :given].float())
        got = torch.cat([pool[0, page] for page in table[:2]], dim=1).float()
        assert torch.equal(got[:, :given], model.x) and got[:, given:].isnan().all()
        got = torch.cat([scale[0, page] for page in table[:2]], dim=1)
        blocks = -(-given // 16)
        assert torch.equal(got[:, :blocks], model.s) and got[:, blocks:].isnan().all()


def test_captured(luvc):
    """Steps of a captured graph give what the calls give."""
    g = torch.Generator(device="cuda").manual_seed(8)
    r = Rig(luvc, 4, 64, 16, 3, 200)
    r.append([0, 1, 2], [rows(g, 1, n, 4, 64) for n in (15, 40, 1)])
    new = torch.zeros((3, 8, 64), dtype=torch.bfloat16, device="cuda")
    back = torch.zeros_like(new)
    one, last = ints([1, 1, 1]), torch.zeros(3, dtype=torch.int32, device="cuda")

    def step():
        last.copy_(r.cache.lengths)
        luvc.kv_reserve(r.cache, one)
        luvc.kv_write(r.cache, new[:, :4], new[:, 4:])
        luvc.kv_read(r.cache, back[:, :4], back[:, 4:], first=last)

    parts = [[rows(g, 1, 1, 4, 64, size=s + 1.0) for _ in range(3)] for s in range(20)]
    graph = None
    for p in parts:
        new.copy_(torch.cat([torch.cat((k[0], v[0]), dim=1) for k, v in p]))
        if graph is None:
            step()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        else:
            graph.replay()
        for slot in range(3):
            for x in range(2):
                r.model[slot][0][x].write(p[slot][x][0].float())
        assert torch.equal(back[:, :4], torch.stack([r.model[s][0][0].rows()[-1] for s in range(3)]).bfloat16())
    r.check()


def test_refusals(luvc):
    pool = torch.zeros((1, 4, 2, 32, 64), device="cuda").to(E4M3)
    scale = torch.zeros((1, 4, 2, 2), device="cuda")
    for bad in (scale[..., :1].contiguous(), scale.half(), scale.cpu(), torch.zeros((1, 4, 2, 32), device="cuda"), None):
        with pytest.raises(ValueError):
            luvc.KvCache(pool, pool.clone(), 2, 2, k_scale=scale, v_scale=bad)
    with pytest.raises(ValueError):
        luvc.KvCache(pool, pool.clone(), 2, 2, k_scale=scale, v_scale=torch.zeros((1, 2), device="cuda"))
    with pytest.raises(ValueError):
        luvc.KvCache(pool.bfloat16(), pool.bfloat16(), 2, 2, k_scale=scale, v_scale=scale)
    c = luvc.KvCache(pool, pool.clone(), 2, 2, k_scale=scale, v_scale=scale.clone())
    assert c.blocks
    k = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(TypeError):
        luvc.kv_read(c, k.float(), k.float())
    with pytest.raises(ValueError):
        luvc.kv_read(c, k, k[:1])
    with pytest.raises(ValueError):
        luvc.kv_read(c, k, k.clone(), first=ints([1]))
    with pytest.raises(luvc.LuvcError):
        luvc.kv_read(c, k, k.clone(), layer=1)
