"""Measured cases of the paged key-value cache and of the attention of one new token over it.

The compressed visual tokens of a request (merged by OIM, pruned by SPU) end as rows of the language
model's key-value cache.  Four operators work on that cache, which lives in pages of a shared pool:

  append    room for new tokens (pages from the pool) and their key and value rows written into it
  compact   after a prune: the kept tokens of a sequence close up into new pages, the old ones go back
  fork      further sequences that share the pages of one (several questions about one image)
  decode    attention of one new token per sequence over its cached tokens

`run` computes them in elementary torch operations in 32 bits, or with the library when `own` is set.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
E4M3_MAX = 448.0


def listed():
    return [
        # one question about one image merged to 64 tokens plus a short text: the smallest call, all latency
        dict(name="decode_image_question", op="decode", dtype="bf16", batch=1, q_heads=28, heads=4, dim=128, page=16,
             shortest=97, longest=97, bias=False),
        # eight high-resolution images pruned to a quarter, with texts of different lengths; merged tokens weigh by
        # their number of sources, as a bias of the scores
        dict(name="decode_pruned_images", op="decode", dtype="bf16", batch=8, q_heads=28, heads=4, dim=128, page=16,
             shortest=340, longest=463, bias=True),
        # eight long videos of up to 16384 tokens that nobody pruned: the largest decode step
        dict(name="decode_videos", op="decode", dtype="bf16", batch=8, q_heads=32, heads=8, dim=128, page=64,
             shortest=4173, longest=16451, bias=False),
        # the same kind of batch, more of it, in an 8-bit cache
        dict(name="decode_videos_8bit", op="decode", dtype="e4m3", batch=12, q_heads=32, heads=8, dim=128, page=64,
             shortest=2601, longest=16451, bias=False),
        # 32-bit cache, every query head with a key head of its own, ragged from an almost empty sequence on
        dict(name="decode_single_precision", op="decode", dtype="f32", batch=6, q_heads=16, heads=16, dim=64, page=16,
             shortest=3, longest=2592, bias=False),
        # a decode step of 32 sequences: one token each, some of which open a page
        dict(name="append_token", op="append", dtype="bf16", batch=32, q_heads=28, heads=4, dim=128, page=16,
             held=700, shortest=1, longest=1, sizes=False),
        # prompts: eight images merged to 1296 tokens with their texts; values are enhanced by log(size)
        dict(name="append_merged_images", op="append", dtype="bf16", batch=8, q_heads=28, heads=4, dim=128, page=16,
             held=0, shortest=1311, longest=1401, sizes=True),
        # prompts of long videos, written to an 8-bit cache
        dict(name="append_videos_8bit", op="append", dtype="e4m3", batch=3, q_heads=32, heads=8, dim=128, page=64,
             held=37, shortest=7001, longest=16384, sizes=False),
        # one image of 1296 tokens pruned to a quarter in the cache of a group of four layers
        dict(name="compact_image", op="compact", dtype="bf16", batch=1, layers=4, heads=4, dim=128, page=16,
             before=14, span=1296, keep=324, after=23),
        # the largest prune: eight videos of 16384 tokens to a quarter
        dict(name="compact_videos", op="compact", dtype="bf16", batch=8, layers=4, heads=8, dim=128, page=64,
             before=21, span=16384, keep=4096, after=75),
        # four questions about one image of 1296 tokens
        dict(name="fork_image", op="fork", dtype="bf16", batch=1, copies=4, layers=4, heads=4, dim=128, page=16,
             shortest=1319, longest=1319),
        # eight samples for each of 32 prompts, a group of seven layers
        dict(name="fork_samples", op="fork", dtype="bf16", batch=32, copies=8, layers=7, heads=4, dim=128, page=16,
             shortest=360, longest=1391),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("decode", "decode", "append", "compact", "fork"))
    dtype = rng.choice(("bf16", "bf16", "f32", "e4m3"))
    size = {"bf16": 2, "f32": 4, "e4m3": 1}[dtype]
    q_heads, heads, dim = rng.choice(((28, 4, 128), (32, 8, 128), (32, 32, 128), (16, 16, 64), (16, 2, 80), (12, 1, 256)))
    page = rng.choice((16, 32, 48, 64, 128))
    c = dict(op=op, dtype=dtype, heads=heads, dim=dim, page=page)
    token = 2 * heads * dim * size
    if op == "decode":
        longest = log(1, 16451)
        batch = max(1, min(log(1, 64), (400 << 20) // (token * longest)))
        c.update(batch=batch, q_heads=q_heads, longest=longest, shortest=rng.randint(0, longest), bias=rng.random() < 0.3)
    elif op == "append":
        longest = log(1, 16384)
        batch = max(1, min(log(1, 64), (100 << 20) // (token * longest)))
        c.update(batch=batch, q_heads=q_heads, held=rng.randint(0, 900), longest=longest, shortest=rng.randint(1, longest),
                 sizes=rng.random() < 0.5)
    elif op == "compact":
        span = log(16, 16384)
        layers = max(1, min(rng.randint(1, 8), (300 << 20) // (token * span)))
        batch = max(1, min(log(1, 16), (400 << 20) // (token * span * layers)))
        c.update(batch=batch, layers=layers, before=rng.randint(0, 90), span=span, keep=rng.randint(1, span),
                 after=rng.randint(0, 300))
    else:
        longest = log(1, 4000)
        layers = rng.randint(1, 8)
        copies = rng.randint(1, 9)
        batch = max(1, min(log(1, 32), (400 << 20) // (token * layers * max(longest, page * (1 + copies)))))
        c.update(batch=batch, copies=copies, layers=layers, longest=longest, shortest=rng.randint(1, longest))
    return c


# ---- sizes that follow from a case alone ------------------------------------------------------


def spread(case, lo, hi, what):
    """One whole number in [lo, hi] per sequence, the same for every seed; the first is the largest."""
    rng = random.Random("%s %d %d %d" % (what, case["batch"], lo, hi))
    return [hi] + [rng.randint(lo, hi) for _ in range(case["batch"] - 1)]


def up(a, b):
    return -(-a // b)


def plan(case):
    """Tokens each sequence holds before the call (slots in use first), pages and table sizes of the pool."""
    n, page = case["batch"], case["page"]
    if case["op"] == "decode":
        held = spread(case, case["shortest"], case["longest"], "length")
        slots, most, fresh = n, case["longest"], 0
    elif case["op"] == "append":
        held = spread(case, case["held"] // 2, case["held"], "held")
        add = spread(case, case["shortest"], case["longest"], "new")
        slots, most = n, max(h + a for h, a in zip(held, add))
        fresh = sum(up(h + a, page) - up(h, page) for h, a in zip(held, add))
    elif case["op"] == "compact":
        first, after = texts(case)
        held = [f + case["span"] + a for f, a in zip(first, after)]
        slots, most = n, max(held)
        fresh = sum(up(f + case["keep"] + a, page) for f, a in zip(first, after))
    else:
        held = spread(case, case["shortest"], case["longest"], "length")
        slots, most, fresh = n * (1 + case["copies"]), case["longest"], n * case["copies"]
    # a pool that is nearly full: what the sequences hold, what the call takes, and an eighth more
    pages = sum(up(h, page) for h in held) + fresh
    return held, slots, up(most, page) + 1, pages + pages // 8 + 4


def texts(case):
    """Tokens before and after the visual block of each sequence."""
    return spread(case, case["before"] // 2, case["before"], "before"), spread(case, case["after"] // 2, case["after"], "after")


def work(case):
    size = {"bf16": 2, "f32": 4, "e4m3": 1}[case["dtype"]]
    wide = 4 if case["dtype"] == "f32" else 2           # queries, outputs and new rows
    held, page = plan(case)[0], case["page"]
    row = case["heads"] * case["dim"]                   # elements of a token's keys in one layer
    entries = 4 * sum(up(h, page) for h in held)
    n = case["batch"]
    if case["op"] == "decode":
        out = n * case["q_heads"] * case["dim"]
        return {"bytes": sum(held) * 2 * row * size + 2 * out * wide + entries + (4 * sum(held) if case["bias"] else 0),
                "flops": 4 * sum(held) * case["q_heads"] * case["dim"]}
    if case["op"] == "append":
        new = sum(spread(case, case["shortest"], case["longest"], "new"))
        return {"bytes": new * 2 * row * (wide + size) + (4 * new if case["sizes"] else 0) + 8 * n, "flops": new * row}
    layers = case["layers"]
    if case["op"] == "compact":
        first, after = texts(case)
        moved = sum(f % page + case["keep"] + a for f, a in zip(first, after))
        return {"bytes": 2 * moved * layers * 2 * row * size + 4 * n * case["keep"] + entries, "flops": 0}
    tails = sum(h % page for h in held) * layers * 2 * row * size
    return {"bytes": tails * (1 + case["copies"]) + entries * (1 + case["copies"]), "flops": 0}


# ---- inputs ------------------------------------------------------------------------------------


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    held, slots, cols, pages = plan(case)
    n, page, heads, dim = case["batch"], case["page"], case["heads"], case["dim"]
    layers, dtype = case.get("layers", 1), TYPES[case["dtype"]]
    wide = torch.float32 if case["dtype"] == "f32" else torch.bfloat16

    def normal(*shape, dtype=wide):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)

    s = dict(case=case, k_scale=None, v_scale=None)
    # keys have channels of a constant offset, values do not; both pools are full of old rows
    offset = 1.5 * normal(layers, 1, heads, 1, dim)
    k = normal(layers, pages, heads, page, dim).add_(offset)
    v = normal(layers, pages, heads, page, dim)
    if case["dtype"] == "e4m3":
        s["k_scale"] = 0.012 + 0.01 * torch.rand((layers, heads), generator=gen, device="cuda")
        s["v_scale"] = 0.008 + 0.01 * torch.rand((layers, heads), generator=gen, device="cuda")
        k = k.div_(s["k_scale"][:, None, :, None, None]).clamp_(-E4M3_MAX, E4M3_MAX).to(dtype)
        v = v.div_(s["v_scale"][:, None, :, None, None]).clamp_(-E4M3_MAX, E4M3_MAX).to(dtype)
    s["k"], s["v"] = k, v
    # pages of the sequences in use lie anywhere in the pool
    order = list(range(pages))
    rng.shuffle(order)
    lengths, refs, table = torch.zeros(slots, dtype=torch.int32), torch.zeros(pages, dtype=torch.int32), torch.full((slots, cols), -1, dtype=torch.int32)
    at = 0
    for b, h in enumerate(held):
        take = order[at:at + up(h, page)]
        at += len(take)
        lengths[b] = h
        table[b, :len(take)] = torch.tensor(take, dtype=torch.int32)
        refs[torch.tensor(take, dtype=torch.long)] = 1
    s["meta"] = torch.cat((lengths, refs, table.reshape(-1))).cuda()
    s["before"] = s["meta"].clone()
    s["lengths"], s["refs"] = s["meta"][:slots], s["meta"][slots:slots + pages]
    s["table"] = s["meta"][slots + pages:].view(slots, cols)
    if case["op"] in ("decode", "append"):
        # queries, keys and values are parts of one projection's output
        hq = case["q_heads"]
        add = spread(case, case["shortest"], case["longest"], "new") if case["op"] == "append" else [1] * n
        qkv = normal(sum(add), hq + 2 * heads, dim)
        qkv[:, hq:hq + heads] += offset[0, :, :, 0]
        s["q"], s["new_k"], s["new_v"] = qkv[:, :hq], qkv[:, hq:hq + heads], qkv[:, hq + heads:]
        s["counts"] = torch.tensor(add, dtype=torch.int32, device="cuda")
        s["starts"] = torch.tensor([sum(add[:i]) for i in range(n + 1)], dtype=torch.int32, device="cuda")
        sizes = torch.randint(1, 10, (sum(add),), generator=gen, device="cuda", dtype=torch.int32)
        s["sizes"] = sizes if case.get("sizes") else None
    if case.get("bias"):
        s["bias"] = torch.randint(1, 10, (n, case["longest"]), generator=gen, device="cuda").float().log()
    if case["op"] == "compact":
        first, after = texts(case)
        s["first"] = torch.tensor(first, dtype=torch.int32, device="cuda")
        s["span"] = torch.full((n,), case["span"], dtype=torch.int32, device="cuda")
        score = torch.rand((n, case["span"]), generator=gen, device="cuda")
        s["idx"] = score.topk(case["keep"], dim=1).indices.sort(dim=1).values.int()
    if case["op"] == "fork":
        s["src"] = torch.arange(n, dtype=torch.int32, device="cuda").repeat_interleave(case["copies"])
        s["dst"] = torch.arange(n, slots, dtype=torch.int32, device="cuda")
        s["parents"] = torch.arange(n, dtype=torch.int32, device="cuda")
    if own:
        import paper_2512_09010_b200 as luvc

        s["cache"] = luvc.KvCache(k, v, slots, cols, meta=s["meta"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    return s


# ---- one pass ----------------------------------------------------------------------------------


def run(s):
    op = s["case"]["op"]
    if op != "decode":
        s["meta"].copy_(s["before"])                    # the pool's books as before the call: the pass starts anew
    return (OWN if own else PLAIN)[op](s)


def state(s):
    return {"k": s["k"], "v": s["v"], "lengths": s["lengths"], "refs": s["refs"], "table": s["table"]}


def own_decode(s):
    import paper_2512_09010_b200 as luvc

    return luvc.attn_decode(s["q"], s["cache"], key_bias=s.get("bias"))


def own_append(s):
    import paper_2512_09010_b200 as luvc

    luvc.kv_reserve(s["cache"], s["counts"])
    luvc.kv_write(s["cache"], s["new_k"], s["new_v"], starts=s["starts"], sizes=s["sizes"])
    return state(s)


def own_compact(s):
    import paper_2512_09010_b200 as luvc

    luvc.kv_compact(s["cache"], s["first"], s["span"], s["idx"])
    return state(s)


def own_fork(s):
    import paper_2512_09010_b200 as luvc

    luvc.kv_fork(s["cache"], s["src"], s["dst"])
    luvc.kv_free(s["cache"], s["parents"])
    return state(s)


OWN = {"decode": own_decode, "append": own_append, "compact": own_compact, "fork": own_fork}


def rows_of(pool):
    """The pool as bytes where its elements have 8 bits (for indexing)."""
    return pool.view(torch.uint8) if pool.dtype == torch.float8_e4m3fn else pool


def plain_decode(s):
    case, page = s["case"], s["case"]["page"]
    n, heads, dim = case["batch"], case["heads"], case["dim"]
    cols = max(1, up(case["longest"], page))
    pages = s["table"][:, :cols].clamp(min=0).long()

    def gather(pool, scale):
        rows = rows_of(pool[0])[pages].view(pool.dtype).float().transpose(1, 2).reshape(n, heads, cols * page, dim)
        return rows if scale is None else rows * scale[0][:, None, None]

    live = (torch.arange(cols * page, device="cuda") < s["lengths"][:, None])[:, None, None]
    score = s["q"].float().reshape(n, heads, -1, dim) * dim ** -0.5 @ gather(s["k"], s["k_scale"]).transpose(2, 3)
    if case["bias"]:
        score[..., :case["longest"]] += s["bias"][:, None, None]
    score = score.masked_fill(~live, -math.inf)
    top = score.amax(3, keepdim=True)
    weight = torch.exp(score - top.masked_fill(top == -math.inf, 0.0))
    total = weight.sum(3, keepdim=True)
    value = gather(s["v"], s["v_scale"]) * live.transpose(2, 3)
    return (weight @ value / total.masked_fill(total == 0, 1.0)).reshape(n, -1, dim).to(s["q"].dtype)


def take_pages(s, have, need):
    """Gives each sequence `need` free pages, the lowest first, for its table's entries from `have` on."""
    free = torch.sort((s["refs"] > 0).int(), stable=True).indices
    at = torch.arange(s["table"].shape[1], device="cuda")
    rank = (need.cumsum(0) - need)[:, None] + at - have[:, None]
    mine = (at >= have[:, None]) & (at < (have + need)[:, None])
    return mine, free[rank.clamp(0, free.numel() - 1)].int()


def move_rows(s, to_page, to_slot, from_page, from_slot):
    rows_of(s["k"])[:, to_page, :, to_slot] = rows_of(s["k"])[:, from_page, :, from_slot]
    rows_of(s["v"])[:, to_page, :, to_slot] = rows_of(s["v"])[:, from_page, :, from_slot]


def plain_append(s):
    case, page = s["case"], s["case"]["page"]
    old = s["lengths"].long()
    new = old + s["counts"]
    have = (old + page - 1) // page
    mine, fresh = take_pages(s, have, (new + page - 1) // page - have)
    s["table"].copy_(torch.where(mine, fresh, s["table"]))
    s["refs"].index_add_(0, fresh[mine].long(), torch.ones_like(fresh[mine]))
    s["lengths"].copy_(new)
    token = torch.arange(s["new_k"].shape[0], device="cuda")
    owner = torch.searchsorted(s["starts"][1:].long(), token, right=True)
    place = old[owner] + token - s["starts"].long()[owner]
    at, slot = s["table"].long()[owner, place // page], place % page
    k, v = s["new_k"].float(), s["new_v"].float()
    if case["sizes"]:
        v = v + s["sizes"].float().log()[:, None, None]
    if case["dtype"] == "e4m3":
        k = (k / s["k_scale"][0][:, None]).clamp(-E4M3_MAX, E4M3_MAX)
        v = (v / s["v_scale"][0][:, None]).clamp(-E4M3_MAX, E4M3_MAX)
    rows_of(s["k"])[0][at, :, slot] = rows_of(k.to(s["k"].dtype))
    rows_of(s["v"])[0][at, :, slot] = rows_of(v.to(s["v"].dtype))
    return state(s)


def plain_compact(s):
    case, page, keep = s["case"], s["case"]["page"], s["case"]["keep"]
    old, table = s["lengths"].long(), s["table"].clone()
    first, span = s["first"].long()[:, None], s["span"].long()[:, None]
    new = old - span[:, 0] + keep
    j = torch.arange(table.shape[1] * page, device="cuda")[None]
    kept = first + s["idx"].long().gather(1, (j - first).clamp(0, keep - 1))
    source = torch.where(j < first, j, torch.where(j < first + keep, kept, j - keep + span))
    # leading full pages whose rows stay where they are are kept, all others are written anew
    still = ((source == j) & (j < new[:, None])).long().cumprod(1).sum(1) // page
    mine, fresh = take_pages(s, still, (new + page - 1) // page - still)
    seq, place = torch.nonzero((j >= still[:, None] * page) & (j < new[:, None]), as_tuple=True)
    origin = source[seq, place]
    move_rows(s, fresh[seq, place // page].long(), place % page, table[seq, origin // page].long(), origin % page)
    at = torch.arange(table.shape[1], device="cuda")
    gone = (at >= still[:, None]) & (table >= 0)
    s["refs"].index_add_(0, fresh[mine].long(), torch.ones_like(fresh[mine]))
    s["refs"].index_add_(0, table[gone].long(), -torch.ones_like(table[gone]))
    s["table"].copy_(torch.where(mine, fresh, torch.where(at < still[:, None], table, -1)))
    s["lengths"].copy_(new)
    return state(s)


def plain_fork(s):
    page, src, dst = s["case"]["page"], s["src"].long(), s["dst"].long()
    length = s["lengths"][src].long()
    full, tail = length // page, length % page
    shared = torch.arange(s["table"].shape[1], device="cuda") < full[:, None]
    mine, fresh = take_pages(s, full, (tail > 0).long())
    old = s["table"][src]
    seq, slot = torch.nonzero(torch.arange(page, device="cuda") < tail[:, None], as_tuple=True)
    move_rows(s, fresh[seq, full[seq]].long(), slot, old[seq, full[seq]].long(), slot)
    taken = torch.where(mine, fresh, torch.where(shared, old, -1))
    s["table"][dst] = taken
    s["refs"].index_add_(0, taken[taken >= 0].long(), torch.ones_like(taken[taken >= 0]))
    s["lengths"][dst] = length.int()
    parents = s["parents"].long()
    gone = s["table"][parents]
    s["refs"].index_add_(0, gone[gone >= 0].long(), -torch.ones_like(gone[gone >= 0]))
    s["table"][parents] = -1
    s["lengths"][parents] = 0
    return state(s)


PLAIN = {"decode": plain_decode, "append": plain_append, "compact": plain_compact, "fork": plain_fork}


# ---- the same in 64 bits, sequence by sequence --------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    held, page = plan(case)[0], case["page"]
    if case["op"] == "decode":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        group = case["q_heads"] // case["heads"]
        for b, h in enumerate(held):
            pages = [int(x) for x in s["table"][b].tolist() if x >= 0]
            for head in range(case["heads"] if h else 0):
                k = torch.cat([s["k"][0, x, head].double() for x in pages])[:h]
                v = torch.cat([s["v"][0, x, head].double() for x in pages])[:h]
                if s["k_scale"] is not None:
                    k, v = k * s["k_scale"][0, head].double(), v * s["v_scale"][0, head].double()
                q = s["q"][b, head * group:(head + 1) * group].double()
                score = torch.einsum("gd,td->gt", q, k) / math.sqrt(case["dim"])
                if case["bias"]:
                    score = score + s["bias"][b, :h].double()
                out[b, head * group:(head + 1) * group] = torch.einsum("gt,td->gd", torch.softmax(score, dim=1), v)
        return out
    if s["k"].numel() > 1 << 28:
        return None
    # the pools hold copies (of new rows, rounded once, where the operator writes new rows)
    pools = {"k": s["k"].double(), "v": s["v"].double()}
    table = [[x for x in row if x >= 0] for row in s["table"].tolist()]
    refs = s["refs"].tolist()

    def lowest_free():
        x = refs.index(0)
        refs[x] = 1
        return x

    if case["op"] == "append":
        add, done = spread(case, case["shortest"], case["longest"], "new"), 0
        for b, h in enumerate(held):
            table[b] += [lowest_free() for _ in range(up(h + add[b], page) - up(h, page))]
            place = torch.arange(h, h + add[b], device="cuda")
            at = torch.tensor(table[b], device="cuda")[place // page]
            k, v = s["new_k"][done:done + add[b]].double(), s["new_v"][done:done + add[b]].double()
            if case["sizes"]:
                v = v + torch.log(s["sizes"][done:done + add[b]].double())[:, None, None]
            if case["dtype"] == "e4m3":
                k = torch.clamp(k / s["k_scale"][0].double()[:, None], -E4M3_MAX, E4M3_MAX)
                v = torch.clamp(v / s["v_scale"][0].double()[:, None], -E4M3_MAX, E4M3_MAX)
            pools["k"][0][at, :, place % page], pools["v"][0][at, :, place % page] = k, v
            done += add[b]
    elif case["op"] == "compact":
        first, idx = texts(case)[0], s["idx"].tolist()
        for b, h in enumerate(held):
            keep = list(range(first[b])) + [first[b] + i for i in idx[b]] + list(range(first[b] + case["span"], h))
            still = 0
            while (still + 1) * page <= len(keep) and keep[(still + 1) * page - 1] == (still + 1) * page - 1:
                still += 1
            new = [lowest_free() for _ in range(up(len(keep), page) - still)]
            place, origin = torch.arange(still * page, len(keep), device="cuda"), torch.tensor(keep[still * page:], dtype=torch.long, device="cuda")
            to = torch.tensor(table[b][:still] + new, dtype=torch.long, device="cuda")[place // page]
            at = torch.tensor(table[b], dtype=torch.long, device="cuda")[origin // page]
            for name in ("k", "v"):
                pools[name][:, to, :, place % page] = pools[name][:, at, :, origin % page]
    else:
        for b, h in enumerate(held):
            for _ in range(case["copies"]):
                if h % page:
                    to, last = lowest_free(), h // page
                    for name in ("k", "v"):
                        pools[name][:, to, :, :h % page] = pools[name][:, table[b][last], :, :h % page]
    return {"k": pools["k"], "v": pools["v"], "lengths": None, "refs": None, "table": None}
