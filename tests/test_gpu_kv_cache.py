"""The paged key-value cache against a plain model of its books and rows: every page number, every reference count and
every row has to be the model's (integers and copies: exact).  Rows that are computed on the way (V + log size, the 8-bit
form) are compared with the definition."""
import numpy as np
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


class Model:
    """The books in plain Python, and for every sequence the id of the token in each position."""

    def __init__(self, pages, page, slots, max_pages):
        self.page, self.max_pages = page, max_pages
        self.refs, self.table, self.ids = [0] * pages, [[] for _ in range(slots)], [[] for _ in range(slots)]

    def take(self):
        p = self.refs.index(0)
        self.refs[p] = 1
        return p

    def reserve(self, slot, ids):
        self.ids[slot] = self.ids[slot] + list(ids)
        while len(self.table[slot]) * self.page < len(self.ids[slot]):
            self.table[slot].append(self.take())

    def fork(self, src, dst):
        full = len(self.ids[src]) // self.page
        self.ids[dst] = list(self.ids[src])
        self.table[dst] = self.table[src][:full]
        if len(self.ids[src]) % self.page:
            self.table[dst].append(self.take())

    def share(self, dst):                       # references of shared pages, counted after every page of the call is taken
        for p in self.table[dst][:len(self.ids[dst]) // self.page]:
            self.refs[p] += 1

    def free(self, slot):
        for p in self.table[slot]:
            self.refs[p] -= 1
        self.table[slot], self.ids[slot] = [], []

    def compact(self, slot, first, span, idx):
        order = list(range(first)) + [first + j for j in idx] + list(range(first + span, len(self.ids[slot])))
        still = 0
        while (still + 1) * self.page <= len(order) and order[(still + 1) * self.page - 1] == (still + 1) * self.page - 1:
            still += 1
        old = self.table[slot][still:]
        self.table[slot] = self.table[slot][:still] + [self.take() for _ in range(-(-len(order) // self.page) - still)]
        self.ids[slot] = [self.ids[slot][j] for j in order]
        return old                              # given back after every page of the call is taken

    def drop(self, pages):
        for p in pages:
            self.refs[p] -= 1


def rows_for(ids, layer, heads, D, kind, dtype):
    """The row of a token id: small whole numbers, exact in every type, different for neighbouring ids, layers, heads, K and V."""
    i = torch.as_tensor(ids, dtype=torch.long, device="cuda")[:, None, None]
    h = torch.arange(heads, device="cuda")[None, :, None]
    d = torch.arange(D, device="cuda")[None, None, :]
    return ((i * 7 + layer * 5 + h * 3 + d + 4 * kind) % 13 - 6).to(dtype)


class Rig:
    def __init__(self, luvc, dtype, pages, page, slots, max_pages, layers=2, heads=2, D=64):
        self.luvc, self.model = luvc, Model(pages, page, slots, max_pages)
        shape = (layers, pages, heads, page, D)
        self.layers, self.heads, self.D, self.dtype = layers, heads, D, TYPES[dtype]
        k = torch.full(shape, float("nan"), device="cuda").to(self.dtype)
        scale = torch.ones((layers, heads), device="cuda") if dtype == "e4m3" else None
        self.cache = luvc.KvCache(k, k.clone(), slots, max_pages, k_scale=scale, v_scale=scale)
        self.next_id = 1

    def ints(self, values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    def append(self, slots, counts):
        self.luvc.kv_reserve(self.cache, self.ints(counts), seqs=self.ints(slots))
        ids = []
        for s, c in zip(slots, counts):
            new = list(range(self.next_id, self.next_id + c))
            self.next_id += c
            self.model.reserve(s, new)
            ids += new
        starts = self.ints(np.concatenate(([0], np.cumsum(counts))))
        for layer in range(self.layers):
            k, v = (rows_for(ids, layer, self.heads, self.D, kind, self.cache.io_dtype) for kind in (0, 1))
            self.luvc.kv_write(self.cache, k, v, layer=layer, starts=starts, seqs=self.ints(slots))

    def check(self):
        assert self.luvc.check_status() == 0
        m, c = self.model, self.cache
        assert c.lengths.tolist() == [len(x) for x in m.ids]
        assert c.refs.tolist() == m.refs
        assert c.table.tolist() == [t + [-1] * (m.max_pages - len(t)) for t in m.table]
        for slot, ids in enumerate(m.ids):
            if not ids:
                continue
            pages = torch.tensor(m.table[slot], device="cuda")
            for layer in range(self.layers):
                for kind, pool in enumerate((c.k, c.v)):
                    got = pool.float()[layer][pages].transpose(1, 2).reshape(-1, self.heads, self.D)[:len(ids)]
                    assert torch.equal(got, rows_for(ids, layer, self.heads, self.D, kind, torch.float32)), (slot, layer, kind)


@pytest.mark.parametrize("dtype,page,D,heads", [("bf16", 16, 64, 2), ("f32", 16, 20, 3), ("e4m3", 32, 80, 1), ("bf16", 48, 128, 7),
                                                ("bf16", 16, 8, 1), ("e4m3", 64, 256, 2)])
def test_a_life_of_appends_forks_prunes_and_frees(luvc, dtype, page, D, heads):
    rng = np.random.default_rng(1234 + page + D)
    r = Rig(luvc, dtype, pages=150, page=page, slots=12, max_pages=9, heads=heads, D=D)
    most = 9 * page
    own = torch.full((luvc.kv_workspace_bytes(r.cache, 12),), 0xAB, dtype=torch.uint8, device="cuda")
    for step in range(40):
        m = r.model
        ws = own if step % 2 else None                           # a caller's workspace needs no preparation
        used = [s for s in range(12) if m.ids[s]]
        empty = [s for s in range(12) if not m.ids[s]]
        what = rng.choice(["append", "fork", "compact", "free"], p=[0.4, 0.2, 0.3, 0.1])
        if what == "append":
            slots = rng.permutation(12)[:rng.integers(1, 7)].tolist()
            counts = [int(min(most - len(m.ids[s]), rng.choice([0, 1, 2, 15, 16, 17, int(rng.integers(0, 3 * page))]))) for s in slots]
            r.append(slots, counts)
        elif what == "fork" and used and empty:
            n = int(rng.integers(1, len(empty) + 1))
            src, dst = rng.choice(used, n).tolist(), rng.permutation(empty)[:n].tolist()
            luvc.kv_fork(r.cache, r.ints(src), r.ints(dst), workspace=ws)
            for s, d in zip(src, dst):
                m.fork(s, d)
            for d in dst:
                m.share(d)
        elif what == "compact" and used:
            slots = rng.permutation(used)[:4].tolist()
            first, span, idx, width = [], [], [], 0
            for s in slots:
                n = len(m.ids[s])
                f = int(rng.integers(0, n + 1))
                sp = int(rng.integers(0, n - f + 1))
                keep = int(rng.choice([0, sp, int(rng.integers(0, sp + 1))]))
                first.append(f), span.append(sp)
                chosen = np.sort(rng.permutation(sp)[:keep])
                if keep and rng.random() < 0.4:                     # a prefix, of which nothing moves
                    chosen = np.arange(keep)
                idx.append(chosen.tolist())
                width = max(width, keep)
            table = torch.full((len(slots), width), 1 << 30, dtype=torch.int32)      # what is past counts[i] is not read
            for row, chosen in zip(table, idx):
                row[:len(chosen)] = torch.tensor(chosen, dtype=torch.int32)
            luvc.kv_compact(r.cache, r.ints(first), r.ints(span), table.cuda(), counts=r.ints([len(x) for x in idx]), seqs=r.ints(slots), workspace=ws)
            old = [m.compact(s, f, sp, x) for s, f, sp, x in zip(slots, first, span, idx)]
            for pages in old:
                m.drop(pages)
        elif what == "free" and used:
            slots = rng.permutation(used)[:2].tolist()
            luvc.kv_free(r.cache, r.ints(slots + slots[:1]))                          # named twice: freed once
            for s in slots:
                m.free(s)
        r.check()


@pytest.mark.parametrize("dtype,page,D,heads,layers", [("e4m3", 16, 16, 37, 3), ("e4m3", 16, 48, 32, 2), ("e4m3", 16, 128, 9, 3), ("bf16", 32, 24, 21, 2),
                                                       ("f32", 16, 28, 16, 3), ("f32", 48, 256, 5, 2)])
def test_short_rows_are_moved_by_teams(luvc, dtype, page, D, heads, layers):
    r = Rig(luvc, dtype, pages=900, page=page, slots=12, max_pages=4000 // page, layers=layers, heads=heads, D=D)
    m = r.model
    r.append([0, 1, 2, 3], [3501, 2000, 31, 1777])
    first, span, keep = [3, 500, 0, 0], [3400, 1490, 31, 1777], [1700, 1489, 30, 888]
    rng = np.random.default_rng(D)
    idx = [np.sort(rng.permutation(n)[:k]).tolist() for n, k in zip(span, keep)]
    table = torch.zeros((4, max(keep)), dtype=torch.int32)
    for row, chosen in zip(table, idx):
        row[:len(chosen)] = torch.tensor(chosen, dtype=torch.int32)
    luvc.kv_compact(r.cache, r.ints(first), r.ints(span), table.cuda(), counts=r.ints(keep), seqs=r.ints([0, 1, 2, 3]))
    for pages in [m.compact(s, f, n, x) for s, f, n, x in zip(range(4), first, span, idx)]:
        m.drop(pages)
    r.check()
    luvc.kv_fork(r.cache, r.ints([0, 0, 1, 2, 3, 3]), r.ints([4, 5, 6, 7, 8, 9]))
    for s, d in zip([0, 0, 1, 2, 3, 3], [4, 5, 6, 7, 8, 9]):
        m.fork(s, d)
    for d in range(4, 10):
        m.share(d)
    r.check()


@pytest.mark.parametrize("pages,slots,held", [(40000, 2100, 500), (8000, 420, 150)])
def test_a_large_pool_and_many_sequences(luvc, pages, slots, held):
    # more pages than one sweep of the scan covers, more sequences than threads of its CTA (first pool), free pages far up
    r = Rig(luvc, "bf16", pages=pages, page=16, slots=slots, max_pages=40, layers=1, heads=1, D=8)
    r.append(list(range(held)), [16 * 40 - 3] * held)
    r.check()
    luvc.kv_free(r.cache, r.ints(list(range(0, held, 7))))
    for s in range(0, held, 7):
        r.model.free(s)
    later = list(range(slots - 1, held - 1, -1))
    for part in (later[:256], later[256:]) if slots < 1000 else (later,):
        r.append(part, [(5 * s) % 37 for s in part])
    r.append(list(range(0, held, 7)), [16 * 20 + 1] * len(range(0, held, 7)))
    r.check()


def test_seqs_may_be_left_out(luvc):
    r = Rig(luvc, "bf16", pages=20, page=16, slots=3, max_pages=4)
    luvc.kv_reserve(r.cache, r.ints([20, 0, 3]))
    for s, c in enumerate([20, 0, 3]):
        r.model.reserve(s, range(100 * s, 100 * s + c))
    ids = r.model.ids[0] + r.model.ids[2]
    for layer in range(2):
        luvc.kv_write(r.cache, *(rows_for(ids, layer, 2, 64, kind, torch.bfloat16) for kind in (0, 1)), layer=layer,
                      starts=r.ints([0, 20, 20, 23]))
    r.check()
    luvc.kv_compact(r.cache, r.ints([2, 0, 0]), r.ints([17, 0, 3]), r.ints([[0, 5], [0, 0], [0, 2]]), counts=r.ints([2, 0, 2]))
    for p in [r.model.compact(0, 2, 17, [0, 5]), r.model.compact(1, 0, 0, []), r.model.compact(2, 0, 3, [0, 2])]:
        r.model.drop(p)
    r.check()


@pytest.mark.parametrize("case", ["pages", "table", "slot", "twice", "negative", "fork full", "fork same", "block", "count"])
def test_what_only_the_device_can_see_leaves_the_cache_as_it_was(luvc, case):
    r = Rig(luvc, "bf16", pages=12, page=16, slots=5, max_pages=6)
    r.append([0, 1], [60, 35])
    before = r.cache.meta.clone()
    i, c = r.ints, r.cache
    word = torch.zeros(4, dtype=torch.int32, device="cuda")
    if case == "pages":           # 7 pages are in use, 5 are free: the first sequence fits, both do not
        luvc.kv_reserve(c, i([48, 48]), seqs=i([2, 3]), device_status=word)
    elif case == "table":
        luvc.kv_reserve(c, i([1, 37]), seqs=i([1, 0]), device_status=word)
    elif case == "slot":
        luvc.kv_reserve(c, i([1, 1]), seqs=i([1, 5]), device_status=word)
    elif case == "twice":
        luvc.kv_reserve(c, i([1, 1]), seqs=i([1, 1]), device_status=word)
    elif case == "negative":
        luvc.kv_reserve(c, i([1, -1]), seqs=i([1, 0]), device_status=word)
    elif case == "fork full":
        luvc.kv_fork(c, i([0, 0]), i([2, 1]), device_status=word)
    elif case == "fork same":
        luvc.kv_fork(c, i([0, 0]), i([2, 2]), device_status=word)
    elif case == "block":
        luvc.kv_compact(c, i([0, 20]), i([60, 16]), i([[0], [1]]), device_status=word)
    else:
        luvc.kv_compact(c, i([0, 20]), i([1, 15]), i([[0, 1], [1, 2]]), device_status=word)
    status = {"pages": 12, "table": 12, "fork full": 3, "block": 4, "count": 4}.get(case, 2)
    luvc.kv_free(c, i([0]), device_status=word)                   # a set word stops the calls that follow
    assert torch.equal(c.meta, before)
    assert luvc.read_status(word) == status
    assert luvc.read_status(word) == 0
    r.append([0, 4], [3, 0])
    r.check()


def test_an_index_outside_its_block_is_replaced_and_reported(luvc):
    r = Rig(luvc, "bf16", pages=12, page=16, slots=2, max_pages=4)
    r.append([0], [40])
    luvc.kv_compact(r.cache, r.ints([4]), r.ints([20]), r.ints([[3, 9, 400]]))
    assert luvc.check_status() == 4
    r.model.drop(r.model.compact(0, 4, 20, [3, 9, 19]))
    r.check()


@pytest.mark.parametrize("tail", [[-5], [-5, 25], [25, 400, 401], [-1 << 31, (1 << 31) - 1]])
def test_an_index_outside_its_block_after_pages_that_stay(luvc, tail):
    # the nearest token inside may lie on a page that is not moved
    r = Rig(luvc, "bf16", pages=12, page=16, slots=2, max_pages=5)
    r.append([0, 1], [70, 5])
    own = torch.full((luvc.kv_workspace_bytes(r.cache, 1),), 0xAB, dtype=torch.uint8, device="cuda")
    luvc.kv_compact(r.cache, r.ints([3]), r.ints([60]), r.ints([list(range(20)) + tail]), workspace=own)
    assert luvc.check_status() == 4
    r.model.drop(r.model.compact(0, 3, 60, list(range(20)) + [min(max(e, 0), 59) for e in tail]))
    r.check()


def test_rows_before_the_sequence_are_not_written(luvc):
    r = Rig(luvc, "bf16", pages=4, page=16, slots=2, max_pages=2)
    r.append([0, 1], [3, 2])
    rows = torch.ones((5, 2, 64), dtype=torch.bfloat16, device="cuda")
    luvc.kv_write(r.cache, rows, rows, layer=0, starts=r.ints([0, 5, 5]))            # five rows, three tokens
    assert luvc.check_status() == 2
    assert bool((r.cache.k[0, r.model.table[0][0], :, :3] == 1).all())
    assert bool(r.cache.k[0, r.model.table[0][0], :, 3:].isnan().all())


@pytest.mark.parametrize("bad", [0, 1777, 2999])
@pytest.mark.parametrize("slot", [-1, 3000, 1 << 30])
def test_a_slot_that_does_not_exist_frees_none_of_the_others(luvc, bad, slot):
    r = Rig(luvc, "bf16", pages=3100, page=16, slots=3000, max_pages=2, layers=1, heads=1, D=8)
    r.append(list(range(3000)), [1 + s % 16 for s in range(3000)])
    before = r.cache.meta.clone()
    seqs = list(range(3000))
    seqs[bad] = slot
    for _ in range(5):
        luvc.kv_free(r.cache, r.ints(seqs))
        assert luvc.check_status() == 2
        assert torch.equal(r.cache.meta, before)
    del seqs[bad]
    luvc.kv_free(r.cache, r.ints(seqs))
    for s in seqs:
        r.model.free(s)
    r.check()


def test_rows_that_cannot_be_placed_leave_the_others_written(luvc):
    n, each, layers = 50, 1000, 3                                        # more rows than run at a time
    r = Rig(luvc, "bf16", pages=n * 63 + 2, page=16, slots=n, max_pages=64, layers=layers, heads=1, D=8)
    slots = list(range(n))
    luvc.kv_reserve(r.cache, r.ints([each] * n))
    for s in slots:
        r.model.reserve(s, range(1 + s * each, 1 + (s + 1) * each))
    starts = r.ints([each * s for s in range(n + 1)])
    ids = sum((r.model.ids[s] for s in slots), [])
    rows = [[rows_for(ids, layer, 1, 8, kind, torch.bfloat16) for kind in (0, 1)] for layer in range(layers)]
    for lost in (0, 7, 49):
        for pool in (r.cache.k, r.cache.v):
            pool.fill_(float("nan"))
        wrong = r.ints(slots)
        wrong[lost] = n
        for layer in range(layers):                                       # a report of a write does not stop the writes of further layers
            luvc.kv_write(r.cache, *rows[layer], layer=layer, starts=starts, seqs=wrong)
        before = r.cache.meta.clone()
        luvc.kv_reserve(r.cache, r.ints([1] * n))                         # but everything else,
        luvc.kv_free(r.cache, r.ints(slots))
        luvc.kv_write(r.cache, rows[0][0] + 1, rows[0][1], starts=starts)  # and then writes too
        assert luvc.check_status() == 2
        assert luvc.check_status() == 0
        assert torch.equal(r.cache.meta, before)
        pages = torch.tensor(r.model.table[lost], device="cuda")
        for pool in (r.cache.k, r.cache.v):
            assert bool(pool[:, pages].isnan().all())
        for layer in range(layers):
            luvc.kv_write(r.cache, *(x[lost * each:(lost + 1) * each] for x in rows[layer]), layer=layer, starts=r.ints([0, each]), seqs=r.ints([lost]))
        r.check()                                                        # every other row was there


@pytest.mark.parametrize("dtype", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("heads,D", [(4, 128), (3, 80), (1, 16)])
def test_written_rows_are_enhanced_and_rounded_once(luvc, dtype, heads, D):
    g = torch.Generator(device="cuda").manual_seed(7)
    counts = [1, 33, 0, 18]
    T, layers = sum(counts), 2
    wide = torch.float32 if dtype == "f32" else torch.bfloat16
    qkv = torch.randn((T, 5 * heads * D), generator=g, device="cuda").to(wide) * 3
    qkv[5, :] *= 1e4                                             # saturates the 8-bit form
    k = qkv[:, 2 * heads * D:3 * heads * D].view(T, heads, D)    # parts of a wider row
    v = qkv[:, 4 * heads * D:].view(T, heads, D)
    sizes = torch.randint(1, 9, (T,), generator=g, device="cuda", dtype=torch.int32)
    scale = (0.5 + torch.rand((layers, heads), generator=g, device="cuda")) * 0.02 if dtype == "e4m3" else None
    pool = torch.zeros((layers, 9, heads, 16, D), device="cuda").to(TYPES[dtype])
    cache = luvc.KvCache(pool, pool.clone(), 4, 4, k_scale=scale, v_scale=scale.flip(0) if scale is not None else None)
    c = torch.tensor(counts, dtype=torch.int32, device="cuda")
    starts = torch.cat((c.new_zeros(1), c.cumsum(0).int()))
    luvc.kv_reserve(cache, c)
    luvc.kv_write(cache, k, v, layer=1, starts=starts, sizes=sizes)
    assert luvc.check_status() == 0
    assert not cache.k[0].float().any()
    got = []
    for p in (cache.k, cache.v):
        rows = [p.float()[1][cache.table[s, :(n + 15) // 16].long()].transpose(1, 2).reshape(-1, heads, D)[:n] for s, n in enumerate(counts) if n]
        got.append(torch.cat(rows))
    want = (k.double(), v.double() + sizes.double().log()[:, None, None])
    if dtype == "e4m3":
        # the quotient in fp32, to the nearest 8-bit value: exact for keys; log's last bit may tip a tie of the values by one step
        q = [(w.float() / s[1][:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).float() for w, s in zip(want, (cache.k_scale, cache.v_scale))]
        assert torch.equal(got[0], q[0])
        assert ((got[1] - q[1]).abs() <= q[1].abs() / 8 + 2.0 ** -9).all() and (got[1] != q[1]).float().mean() < 1e-3
        assert got[0].abs().max() == 448
    else:
        assert torch.equal(got[0].double(), want[0])
        # unit roundoff of the type, and log's and the sum's rounding in fp32
        u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
        assert ((got[1].double() - want[1]).abs() <= u * want[1].abs() + 4 * 2.0 ** -24 * (v.double().abs() + 3)).all()


def test_every_bf16_value_is_divided_as_a_division_does(luvc):
    """All 65536 bf16 patterns (subnormals, infinities and NaN among them) over scales that give ties, quotients that saturate, and
    reciprocals that overflow: the stored byte is that of the nearest 8-bit value to the fp32 quotient."""
    scales = [1.0, 0.75, 1.5, 3.0, 7.0, 0.1, 0.013, 1 / 3, 2.0 ** -20, 2.0 ** -126, 2.0 ** -130, 2.0 ** -149, 2.0 ** 100, 3e38, 1e-5, 448.0]
    heads, D, tokens = len(scales), 64, 1024
    x = torch.arange(65536, dtype=torch.int32, device="cuda").to(torch.int16).view(torch.bfloat16).view(tokens, 1, D)
    x = x.expand(tokens, heads, D).contiguous()
    s = torch.tensor([scales], device="cuda")
    pool = torch.zeros((1, tokens // 64, heads, 64, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    cache = luvc.KvCache(pool, pool.clone(), 1, tokens // 64, k_scale=s, v_scale=s.flip(1))
    count = torch.tensor([tokens], dtype=torch.int32, device="cuda")
    luvc.kv_reserve(cache, count)
    luvc.kv_write(cache, x, x, starts=torch.tensor([0, tokens], dtype=torch.int32, device="cuda"))
    assert luvc.check_status() == 0
    for got, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        want = (x.float() / scale[0][:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).float()
        have = got.float()[0].transpose(1, 2).reshape(tokens, heads, D)
        same = (have == want) | (have.isnan() & want.isnan())
        assert bool(same.all()), (x[~same][:5], have[~same][:5], want[~same][:5])


def test_a_step_can_be_captured_and_replayed(luvc):
    """A decode step (room, rows, attention) in a CUDA graph: page numbers are worked out on the device at every replay."""
    r = Rig(luvc, "bf16", pages=16, page=16, slots=2, max_pages=5, layers=1)
    r.append([0, 1], [14, 3])
    c, one = r.cache, r.ints([1, 1])
    k = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")       # equal scores: the mean of the values
    out = torch.empty_like(q)
    word = torch.zeros(4, dtype=torch.int32, device="cuda")
    ws = torch.zeros(luvc.attn_workspace_bytes(), dtype=torch.uint8, device="cuda")

    def step():
        luvc.kv_reserve(c, one, device_status=word)
        luvc.kv_write(c, k, v, device_status=word)
        luvc.attn_decode(q, c, out=out, workspace=ws, device_status=word)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        luvc.kv_write(c, k, v, device_status=word)                         # loads the kernels; rewritten below
        luvc.attn_decode(q, c, out=out, workspace=ws, device_status=word)
        luvc.kv_reserve(c, r.ints([0, 0]), device_status=word)
    side.synchronize()
    for s in (0, 1):                                                       # the rows the warm-up overwrote
        last = r.model.ids[s][-1:]
        kk, vv = (rows_for(last, 0, 2, 64, kind, torch.bfloat16) for kind in (0, 1))
        luvc.kv_write(c, kk, vv, seqs=r.ints([s]))
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(20):
        ids = [r.next_id, r.next_id + 1]
        r.next_id += 2
        for s in (0, 1):
            r.model.reserve(s, [ids[s]])
        k.copy_(rows_for(ids, 0, 2, 64, 0, torch.bfloat16))
        v.copy_(rows_for(ids, 0, 2, 64, 1, torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        for s in (0, 1):
            mean = rows_for(r.model.ids[s], 0, 2, 64, 1, torch.float64).mean(0).repeat_interleave(2, 0)
            assert ((out[s].double() - mean).abs() <= 2.0 ** -8 * mean.abs() + 1e-5).all()
    assert luvc.read_status(word) == 0
    r.check()


def test_a_captured_fork_keeps_its_scratch(luvc):
    """The library's scratch grows for a call that needs more; a graph captured before goes on with the memory it was captured with."""
    luvc.shutdown()                                                        # scratch starts small
    r = Rig(luvc, "bf16", pages=40, page=16, slots=6, max_pages=5)
    r.append([0, 1], [40, 21])
    src, dst = r.ints([0, 1, 0]), r.ints([2, 3, 4])

    def step():
        luvc.kv_fork(r.cache, src, dst)
        luvc.kv_compact(r.cache, zero, span, idx, seqs=dst)
        luvc.kv_free(r.cache, dst)

    zero, span, idx = r.ints([0] * 3), r.ints([17] * 3), r.ints([[1, 4, 16]] * 3)
    step()                                                                 # grows the scratch, loads the kernels
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step()
    big = Rig(luvc, "bf16", pages=4000, page=16, slots=400, max_pages=5000, layers=1, heads=1, D=8)
    big.append([0], [77])
    luvc.kv_fork(big.cache, big.ints([0] * 399), big.ints(list(range(1, 400))))
    for d in range(1, 400):
        big.model.fork(0, d)
    for d in range(1, 400):
        big.model.share(d)
    big.check()
    # what a freed scratch would be given to: its contents are looked at after the replays
    fill = [torch.full((1 << 16,), 0x5a5a5a5a, dtype=torch.int32, device="cuda") for _ in range(64)]
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    r.check()
    big.check()
    assert all(bool((f == 0x5a5a5a5a).all()) for f in fill)
    luvc.kv_fork(r.cache, src, dst)
    for s, d in ((0, 2), (1, 3), (0, 4)):
        r.model.fork(s, d)
    for d in (2, 3, 4):
        r.model.share(d)
    r.check()


def test_threads_with_few_and_many_sequences(luvc):
    """Calls of different size from two host threads at once, each on its own cache, stream and status block (the plan's shared
    memory depends on the number of sequences)."""
    import threading

    failed = []

    def work(n):
        try:
            r = Rig(luvc, "bf16", pages=8, page=16, slots=n, max_pages=2, layers=1, heads=1, D=8)
            word, zero, slots = torch.zeros(4, dtype=torch.int32, device="cuda"), r.ints([0] * n), r.ints(list(range(n)))
            torch.cuda.synchronize()
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(3000):
                    luvc.kv_reserve(r.cache, zero, seqs=slots, device_status=word)
            torch.cuda.synchronize()
            assert luvc.read_status(word) == 0
        except Exception as e:                                            # noqa: BLE001
            failed.append((n, e))

    threads = [threading.Thread(target=work, args=(n,)) for n in (1000, 4096, 1500, 3000)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed


def test_python_refusals(luvc):
    pool = torch.zeros((1, 4, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(TypeError):
        luvc.KvCache(pool.half(), pool.half(), 2, 2)
    with pytest.raises(ValueError):
        luvc.KvCache(pool, pool[:, :3], 2, 2)
    with pytest.raises(ValueError):
        luvc.KvCache(pool.cpu(), pool.cpu(), 2, 2)
    with pytest.raises(ValueError):
        luvc.KvCache(pool, pool.clone(), 2, 2, meta=torch.zeros(9, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        luvc.KvCache(pool, pool.clone(), 2, 2, k_scale=torch.ones((1, 2), device="cuda"), v_scale=torch.ones((1, 2), device="cuda"))
    with pytest.raises(ValueError):
        luvc.KvCache(pool.to(torch.float8_e4m3fn), pool.to(torch.float8_e4m3fn), 2, 2)
    c = luvc.KvCache(pool, pool.clone(), 2, 2)
    with pytest.raises(ValueError):
        luvc.kv_reserve(c, torch.ones(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        luvc.kv_reserve(c, torch.ones(2, dtype=torch.int32))
    row = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(TypeError):
        luvc.kv_write(c, row.float(), row.float())
    with pytest.raises(ValueError):
        luvc.kv_write(c, row.transpose(1, 2).contiguous().transpose(1, 2), row)
    with pytest.raises(luvc.LuvcError) as e:
        luvc.kv_write(c, row, row, layer=1)
    assert e.value.status == 2
    with pytest.raises(ValueError):
        luvc.attn_decode(row[..., :32], c)
    with pytest.raises(ValueError):
        luvc.attn_decode(row, c, key_bias=torch.zeros((1, 4), device="cuda"))
    with pytest.raises(luvc.LuvcError) as e:
        luvc.attn_decode(torch.zeros((2, 3, 64), dtype=torch.bfloat16, device="cuda"), c)
    assert e.value.status == 2


def test_workspaces_and_status_blocks_elsewhere_are_refused(luvc):
    """Memory that the kernels cannot reach, or that is shorter than they take it for, is refused before anything is queued."""
    pool = torch.zeros((1, 4, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    c = luvc.KvCache(pool, pool.clone(), 2, 2)
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    row = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    calls = (lambda **o: luvc.kv_fork(c, one - 1, one, **o), lambda **o: luvc.kv_compact(c, one - 1, one - 1, one[None] - 1, **o),
             lambda **o: luvc.attn_decode(row, c, **o))
    size = luvc.attn_workspace_bytes()
    for call in calls:
        for bad in (torch.zeros(size, dtype=torch.uint8), torch.zeros((size // 256, 512), dtype=torch.uint8, device="cuda")[:, :256]):
            with pytest.raises(ValueError):
                call(workspace=bad)
        with pytest.raises(luvc.LuvcError) as e:
            call(workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))
        assert e.value.status == 8
    calls += (lambda **o: luvc.kv_reserve(c, one, **o), lambda **o: luvc.kv_write(c, row, row, **o), lambda **o: luvc.kv_free(c, one, **o))
    for call in calls:
        for bad in (torch.zeros(4, dtype=torch.int32), torch.zeros(4, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"),
                    torch.zeros(8, dtype=torch.int32, device="cuda")[::2]):
            with pytest.raises(ValueError):
                call(device_status=bad)
    assert luvc.check_status() == 0 and not c.meta[:6].any()


def test_a_lone_token_may_have_any_stride(luvc):
    r = Rig(luvc, "bf16", pages=4, page=16, slots=1, max_pages=2, layers=1)
    r.append([0], [20])
    luvc.kv_reserve(r.cache, r.ints([1]))
    r.model.reserve(0, [r.next_id])
    rows = [torch.zeros((3, 129), dtype=torch.bfloat16, device="cuda")[:, :128].view(3, 2, 64)[:1] for _ in range(2)]   # 129 elements to the next row
    for kind in (0, 1):
        rows[kind].copy_(rows_for([r.next_id], 0, 2, 64, kind, torch.bfloat16))
    assert rows[0].stride(0) == 129
    luvc.kv_write(r.cache, *rows)
    r.check()
    q = torch.randn((2, 257), device="cuda").bfloat16()[:, :256].view(2, 4, 64)[:1]
    assert q.stride(0) == 257 and torch.equal(luvc.attn_decode(q, r.cache), luvc.attn_decode(q.contiguous(), r.cache))


def test_the_largest_write(luvc):
    # 2^31 - 16 tokens of one head of 8 (32 GB) in one call: the number of CTAs is counted without overflow
    if torch.cuda.mem_get_info()[0] < 110 << 30:
        pytest.skip("needs 110 GB")
    pages, n = (1 << 27) - 1, (1 << 31) - 16
    pool = torch.zeros((1, pages, 1, 16, 8), dtype=torch.bfloat16, device="cuda")
    c = luvc.KvCache(pool, torch.zeros_like(pool), 1, pages)
    rows = torch.empty((n, 1, 8), dtype=torch.bfloat16, device="cuda")
    rows.view(torch.int32).random_(generator=torch.Generator(device="cuda").manual_seed(3)).bitwise_and_(-1077952577)     # 0xbfbfbfbf: finite
    for count in (1 << 30, n - (1 << 30)):
        luvc.kv_reserve(c, torch.tensor([count], dtype=torch.int32, device="cuda"))
    luvc.kv_write(c, rows, rows, starts=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    assert luvc.check_status() == 0
    assert int(c.lengths[0]) == n and c.table[0, :3].tolist() == [0, 1, 2] and int(c.table[0, -1]) == pages - 1
    want = rows.view(-1).view(torch.int64)
    for got in (c.k, c.v):                                        # the pages were handed out in order
        for a, b in zip(got.view(-1).view(torch.int64).split(1 << 28), want.split(1 << 28)):
            assert torch.equal(a, b)
    del c, pool, rows, want, got, a, b
    torch.cuda.empty_cache()
