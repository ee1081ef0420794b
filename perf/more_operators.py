"""Measured cases of what stands between a projection and an answer: rotary positions, a block-scaled 8-bit cache, and the
attention over it and over an encoder's states.

  rope     the queries and keys of new tokens turned by their positions (one number each, or frame, row and column of the
           patch grid), and the turn back that the backward pass and a change of position need
  write    keys and values quantised on their way into a paged cache of 8 bits, one scale for each 16 tokens of a head that
           follows from the rows
  read     rows of that cache back as 16-bit rows, for an operator that wants them dense
  decode   attention of one new token per sequence over that cache
  cross    attention of a text's tokens to the merged visual tokens of its image or video, which have no order among
           themselves: no causal mask, and merged tokens weigh by log(size)

`run` computes them in elementary torch operations in 32 bits, or with the library when `own` is set.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E4M3_MAX = 448.0
BLOCK = 16                  # tokens that share a scale
LEAST, MOST = -60, 60       # exponents a scale may have


def listed():
    return [
        # a decode step of 32 sequences: queries and keys of one token each, in place in the fused projection's row
        dict(name="rope_step", op="rope", dtype="bf16", tokens=32, heads=32, behind=4, dim=128, rotary=128, axes=1,
             interleaved=False, inverse=False, far=16451),
        # prompts of long videos: positions are (frame, row, column), each for its own part of the frequencies
        dict(name="rope_video_prompts", op="rope", dtype="bf16", tokens=16384, heads=40, behind=8, dim=128, rotary=128, axes=3,
             interleaved=False, inverse=False, far=128),
        # backward pass of interleaved pairs in half of a head, 32 bits, positions of a long context with stretched frequencies
        dict(name="rope_backward_long_context", op="rope", dtype="f32", tokens=4999, heads=32, behind=0, dim=80, rotary=40, axes=1,
             interleaved=True, inverse=True, far=1 << 20),
        # a decode step: one token for each of 32 sequences, most into a block that is in use
        dict(name="write_step", op="write", batch=32, heads=4, dim=128, page=16, held=700, shortest=1, longest=1, sizes=False),
        # prompts of long videos whose tokens were merged: values are enhanced by log(size), then quantised
        dict(name="write_video_prompts", op="write", batch=3, heads=8, dim=128, page=64, held=37, shortest=7001, longest=16384, sizes=True),
        # the same prompts read back for another operator
        dict(name="read_video_prompts", op="read", batch=3, heads=8, dim=128, page=64, shortest=7001, longest=16384),
        # one question about one image merged to 64 tokens plus a short text: the smallest call, all latency
        dict(name="decode_image_question", op="decode", batch=1, q_heads=28, heads=4, dim=128, page=16, shortest=97, longest=97, bias=False),
        # twelve long videos
        dict(name="decode_videos", op="decode", batch=12, q_heads=32, heads=8, dim=128, page=64, shortest=2601, longest=16451, bias=False),
        # one new token for each of 16 texts, to the tokens of its image: merged to at most 1296, pruned to a quarter at least
        dict(name="cross_step", op="cross", dtype="bf16", batch=16, q_heads=28, heads=4, dim=128, q_shortest=1, q_longest=1,
             k_shortest=324, k_longest=1296, bias=True),
        # eight questions about images merged to 1296 tokens
        dict(name="cross_questions", op="cross", dtype="bf16", batch=8, q_heads=28, heads=4, dim=128, q_shortest=17, q_longest=96,
             k_shortest=1296, k_longest=1296, bias=True),
        # two long texts to the tokens of a video that nobody pruned: all products
        dict(name="cross_videos", op="cross", dtype="bf16", batch=2, q_heads=32, heads=8, dim=128, q_shortest=1777, q_longest=2048,
             k_shortest=12001, k_longest=16384, bias=False),
        # 32 bits, every head with keys of its own, grids of 24 by 24 merged to different degrees
        dict(name="cross_single_precision", op="cross", dtype="f32", batch=6, q_heads=16, heads=16, dim=64, q_shortest=33, q_longest=257,
             k_shortest=64, k_longest=576, bias=True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("rope", "write", "read", "decode", "cross", "cross"))
    q_heads, heads, dim = rng.choice(((28, 4, 128), (32, 8, 128), (32, 32, 128), (16, 16, 64), (16, 2, 80), (12, 1, 256)))
    page = rng.choice((16, 32, 48, 64, 128))
    if op == "rope":
        dtype = rng.choice(("bf16", "bf16", "f32"))
        size = 2 if dtype == "bf16" else 4
        most = (160 << 20) // (size * dim * (q_heads + 2 * heads))
        return dict(op=op, dtype=dtype, tokens=log(1, most), heads=q_heads + heads, behind=heads, dim=dim,
                    rotary=rng.choice((dim, dim, dim // 2, dim // 4)), axes=rng.choice((1, 1, 3)), interleaved=rng.random() < 0.4,
                    inverse=rng.random() < 0.3, far=log(16, 1 << 20))
    if op in ("write", "read"):
        longest = log(1, 16384)
        batch = max(1, min(log(1, 64), (96 << 20) // (2 * heads * dim * longest)))
        c = dict(op=op, batch=batch, heads=heads, dim=dim, page=page, shortest=rng.randint(1, longest), longest=longest)
        if op == "write":
            c.update(held=rng.randint(0, 900), sizes=rng.random() < 0.5)
        return c
    if op == "decode":
        longest = log(1, 16451)
        batch = max(1, min(log(1, 64), (280 << 20) // (2 * heads * dim * longest)))
        return dict(op=op, batch=batch, q_heads=q_heads, heads=heads, dim=dim, page=page, shortest=rng.randint(0, longest), longest=longest,
                    bias=rng.random() < 0.3)
    dtype = rng.choice(("bf16", "bf16", "f32"))
    k_longest, q_longest = log(1, 16384), rng.choice((1, log(1, 2048), log(1, 2048)))
    flops = 4 * q_heads * dim * q_longest * k_longest
    most = 9e11 if dtype == "bf16" else 3e10
    if flops > most:
        q_longest = max(1, int(q_longest * most / flops))
        flops = 4 * q_heads * dim * q_longest * k_longest
    rows = (2 * heads * k_longest + 2 * q_heads * q_longest) * dim * (2 if dtype == "bf16" else 4)
    batch = int(max(1, min(log(1, 64), most // flops, (400 << 20) // rows)))
    return dict(op=op, dtype=dtype, batch=batch, q_heads=q_heads, heads=heads, dim=dim, q_shortest=rng.randint(1, q_longest), q_longest=q_longest,
                k_shortest=rng.randint(0, k_longest), k_longest=k_longest, bias=rng.random() < 0.5)


# ---- sizes that follow from a case alone ------------------------------------------------------


def spread(case, lo, hi, what):
    """One whole number in [lo, hi] per sequence, the same for every seed; the first is the largest."""
    rng = random.Random("%s %d %d %d" % (what, case["batch"], lo, hi))
    return [hi] + [rng.randint(lo, hi) for _ in range(case["batch"] - 1)]


def starts_of(counts):
    return [sum(counts[:i]) for i in range(len(counts) + 1)]


def up(a, b):
    return -(-a // b)


def plan(case):
    """Tokens each sequence holds before the call, and those the call adds."""
    if case["op"] == "write":
        return spread(case, case["held"] // 2, case["held"], "held"), spread(case, case["shortest"], case["longest"], "new")
    return spread(case, case["shortest"], case["longest"], "length"), [0] * case["batch"]


def work(case):
    op = case["op"]
    if op == "rope":
        size = 2 if case["dtype"] == "bf16" else 4
        turned = case["tokens"] * case["heads"]
        return {"bytes": 2 * turned * case["dim"] * size + 4 * case["tokens"] * case["axes"], "flops": 3 * turned * case["rotary"]}
    n, row = case["batch"], case.get("heads", 0) * case["dim"]
    if op == "cross":
        size = 2 if case["dtype"] == "bf16" else 4
        queries = spread(case, case["q_shortest"], case["q_longest"], "queries")
        keys = spread(case, case["k_shortest"], case["k_longest"], "keys")
        pairs = sum(a * b for a, b in zip(queries, keys))
        return {"bytes": 2 * sum(keys) * row * size + 2 * sum(queries) * case["q_heads"] * case["dim"] * size
                + (4 * sum(keys) if case["bias"] else 0), "flops": 4 * pairs * case["q_heads"] * case["dim"]}
    held, add = plan(case)
    scales = lambda tokens: 8 * case["heads"] * sum(up(t, BLOCK) for t in tokens)                # noqa: E731
    if op == "write":
        return {"bytes": sum(add) * 2 * row * 3 + (4 * sum(add) if case["sizes"] else 0) + scales(add), "flops": 2 * sum(add) * row}
    if op == "read":
        return {"bytes": sum(held) * 2 * row * 3 + scales(held), "flops": sum(held) * 2 * row}
    out = n * case["q_heads"] * case["dim"]
    return {"bytes": sum(held) * 2 * row + 4 * out + scales(held) + 4 * sum(up(h, case["page"]) for h in held)
            + (4 * sum(held) if case["bias"] else 0), "flops": 4 * sum(held) * case["q_heads"] * case["dim"]}


# ---- inputs ------------------------------------------------------------------------------------


def frequencies(rotary, far):
    """Radians per position; stretched, where positions go beyond a context of 32768 tokens, by a larger base."""
    base = 10000.0 * max(1.0, far / 32768.0) ** (rotary / max(1, rotary - 2))
    return (base ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / rotary)).float()


def quantise(x, sizes=None):
    """[..., tokens, D] to e4m3 and a scale for each 16 tokens: the smallest power of two that takes the block's range."""
    y = x.float().unflatten(-2, (-1, BLOCK))
    mantissa, exponent = torch.frexp(y.abs().amax((-2, -1)))                    # 448 = 0.875 * 2^9
    exponent = torch.where(mantissa <= 0.875, exponent - 9, exponent - 8).clamp(LEAST, MOST)
    exponent = torch.where(mantissa == 0.0, torch.full_like(exponent, LEAST), exponent)
    scale = torch.ldexp(torch.ones_like(mantissa), exponent)
    y = (y / scale[..., None, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return y.flatten(-3, -2), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    op, dim, heads = case["op"], case["dim"], case["heads"]
    dtype = TYPES[case.get("dtype", "bf16")]

    def normal(*shape, dtype=dtype):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    s = dict(case=case)
    if op == "rope":
        tokens, axes, half = case["tokens"], case["axes"], case["rotary"] // 2
        s["x"] = normal(tokens, heads + case["behind"], dim)[:, :heads]
        shape = (axes, tokens) if axes > 1 else (tokens,)
        s["positions"] = torch.randint(0, case["far"], shape, generator=gen, device="cuda", dtype=torch.int32)
        s["freqs"] = frequencies(case["rotary"], case["far"]).cuda()
        # a quarter of the frequencies for the frame, three eighths each for row and column
        first, second = half // 4, half // 4 + (half - half // 4) // 2
        s["axis"] = ints([0 if i < first else 1 if i < second else 2 for i in range(half)]) if axes > 1 else None
        return s
    n = case["batch"]
    if op == "cross":
        queries = spread(case, case["q_shortest"], case["q_longest"], "queries")
        keys = spread(case, case["k_shortest"], case["k_longest"], "keys")
        s["queries"], s["keys"] = queries, keys
        s["q"] = normal(sum(queries), case["q_heads"], dim)
        # keys and values are parts of one projection's output; keys have channels of a constant offset
        kv = normal(sum(keys), 2 * heads, dim)
        kv[:, :heads] += 1.5 * normal(heads, dim)
        s["k"], s["v"] = kv[:, :heads], kv[:, heads:]
        s["q_starts"], s["k_starts"] = ints(starts_of(queries)), ints(starts_of(keys))
        s["bias"] = torch.randint(1, 10, (sum(keys),), generator=gen, device="cuda").float().log() if case["bias"] else None
        return s
    page = case["page"]
    held, add = plan(case)
    cols = max(up(h + a, page) for h, a in zip(held, add)) + 1
    pages = sum(up(h + a, page) for h, a in zip(held, add))
    pages += pages // 8 + 4
    # keys have channels of a constant offset; tokens differ in the length of their values, the first ones have short ones
    offset = 1.5 * normal(1, heads, 1, dim)
    k = normal(pages, heads, page, dim).add_(offset)
    v = normal(pages, heads, page, dim)
    v *= torch.exp(0.5 * normal(pages, 1, page, 1, dtype=torch.float32)).to(dtype)
    order = list(range(pages))
    rng.shuffle(order)
    lengths, refs, table = torch.zeros(n, dtype=torch.int32), torch.zeros(pages, dtype=torch.int32), torch.full((n, cols), -1, dtype=torch.int32)
    at = 0
    for b, h in enumerate(held):
        take = order[at:at + up(h, page)]
        at += len(take)
        lengths[b] = h
        table[b, :len(take)] = torch.tensor(take, dtype=torch.int32)
        refs[torch.tensor(take, dtype=torch.long)] = 1
        if take:
            v[take[0], :, :2] *= 0.05
    (k, k_scale), (v, v_scale) = quantise(k[None]), quantise(v[None])
    s.update(k=k, v=v, k_scale=k_scale, v_scale=v_scale)
    s["meta"] = torch.cat((lengths, refs, table.reshape(-1))).cuda()
    s["before"] = s["meta"].clone()
    s["lengths"], s["refs"], s["table"] = s["meta"][:n], s["meta"][n:n + pages], s["meta"][n + pages:].view(n, cols)
    if op == "write":
        kv = normal(sum(add), 2 * heads, dim)
        kv[:, :heads] += offset[0, :, 0]
        s["new_k"], s["new_v"] = kv[:, :heads], kv[:, heads:]
        s["counts"], s["starts"] = ints(add), ints(starts_of(add))
        s["sizes"] = torch.randint(1, 10, (sum(add),), generator=gen, device="cuda", dtype=torch.int32) if case["sizes"] else None
    elif op == "read":
        s["starts"] = ints(starts_of(held))
        s["rows_k"], s["rows_v"] = torch.empty((2, sum(held), heads, dim), dtype=dtype, device="cuda")
    else:
        s["q"] = normal(n, case["q_heads"] + 2 * heads, dim)[:, :case["q_heads"]]
        s["bias"] = torch.randint(1, 10, (n, case["longest"]), generator=gen, device="cuda").float().log() if case["bias"] else None
    if own:
        import paper_2512_09010_b200 as luvc

        s["cache"] = luvc.KvCache(s["k"], s["v"], n, cols, meta=s["meta"], k_scale=k_scale, v_scale=v_scale)
    return s


# ---- one pass ----------------------------------------------------------------------------------


def run(s):
    op = s["case"]["op"]
    if op == "write":
        s["meta"].copy_(s["before"])                    # the pool's books as before the call: the pass starts anew
    return (OWN if own else PLAIN)[op](s)


def written(s):
    return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"], "lengths": s["lengths"], "refs": s["refs"],
            "table": s["table"]}


def own_rope(s):
    import paper_2512_09010_b200 as luvc

    return luvc.rope(s["x"], s["positions"], s["freqs"], axis=s["axis"], interleaved=s["case"]["interleaved"], inverse=s["case"]["inverse"])


def own_write(s):
    import paper_2512_09010_b200 as luvc

    luvc.kv_reserve(s["cache"], s["counts"])
    luvc.kv_write(s["cache"], s["new_k"], s["new_v"], starts=s["starts"], sizes=s["sizes"])
    return written(s)


def own_read(s):
    import paper_2512_09010_b200 as luvc

    luvc.kv_read(s["cache"], s["rows_k"], s["rows_v"], starts=s["starts"])
    return s["rows_k"], s["rows_v"]


def own_decode(s):
    import paper_2512_09010_b200 as luvc

    return luvc.attn_decode(s["q"], s["cache"], key_bias=s["bias"])


def own_cross(s):
    import paper_2512_09010_b200 as luvc

    return luvc.attn_cross(s["q"], s["k"], s["v"], q_starts=s["q_starts"], k_starts=s["k_starts"], key_bias=s["bias"])


OWN = {"rope": own_rope, "write": own_write, "read": own_read, "decode": own_decode, "cross": own_cross}


def plain_rope(s):
    case, x = s["case"], s["x"].float()
    half = case["rotary"] // 2
    where = s["positions"] if s["axis"] is None else s["positions"][s["axis"].long()].t()
    angle = where.double().view(x.shape[0], -1) * s["freqs"].double()             # far positions: 32 bits lose the angle
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if case["inverse"]:
        sin = -sin
    out = x.clone()
    if case["interleaved"]:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        out[..., 0:2 * half:2], out[..., 1:2 * half:2] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        out[..., :half], out[..., half:2 * half] = a * cos - b * sin, a * sin + b * cos
    return out.to(s["x"].dtype)


def bytes_of(pool):
    return pool.view(torch.uint8)                       # (8-bit floats are not indexed as they are)


def block_rows(pool, scale, page, slot):
    """Rows (page, every head, slot) of a layer as 32-bit values."""
    x = bytes_of(pool)[0][page, :, slot].view(pool.dtype).float()
    return x * scale[0][page, :, slot // BLOCK][..., None]


def plain_write(s):
    case, page = s["case"], s["case"]["page"]
    n, cols = s["table"].shape
    old = s["lengths"].long()
    new = old + s["counts"]
    have, need = (old + page - 1) // page, (new + page - 1) // page - (old + page - 1) // page
    free = torch.sort((s["refs"] > 0).int(), stable=True).indices
    at = torch.arange(cols, device="cuda")
    rank = (need.cumsum(0) - need)[:, None] + at - have[:, None]
    mine = (at >= have[:, None]) & (at < (have + need)[:, None])
    fresh = free[rank.clamp(0, free.numel() - 1)].int()
    s["table"].copy_(torch.where(mine, fresh, s["table"]))
    s["refs"].index_add_(0, fresh[mine].long(), torch.ones_like(fresh[mine]))
    s["lengths"].copy_(new)
    # all rows of the blocks the call writes to: the old ones as they are, the new ones
    first, last = old // BLOCK, (new + BLOCK - 1) // BLOCK
    blocks = torch.where(s["counts"] > 0, last - first, torch.zeros_like(first))
    owner = torch.repeat_interleave(torch.arange(n, device="cuda"), blocks)
    block = first[owner] + torch.arange(owner.numel(), device="cuda") - (blocks.cumsum(0) - blocks)[owner]
    place = block[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")                  # [blocks, 16]
    is_new = (place >= old[owner, None]) & (place < new[owner, None])
    is_old = place < old[owner, None]
    source = (s["starts"].long()[owner, None] + place - old[owner, None]).clamp(0, s["new_k"].shape[0] - 1)
    to = s["table"].long()[owner, block * BLOCK // page]
    slot = place % page
    for name in ("k", "v"):
        pool, scale = s[name], s[name + "_scale"]
        rows = s["new_" + name].float()
        if name == "v" and case["sizes"]:
            rows = rows + s["sizes"].float().log()[:, None, None]
        rows = rows[source] * is_new[..., None, None]                                    # [blocks, 16, heads, D]
        before = bytes_of(pool)[0][to[:, None], :, slot]
        _, fits = quantise(rows.transpose(1, 2))                                         # [blocks, heads, 1]
        was = scale[0][to, :, slot[:, 0] // BLOCK]                                       # [blocks, heads]
        now = torch.where(is_old[:, :1], torch.maximum(was, fits[..., 0]), fits[..., 0])
        kept = (before.view(pool.dtype).float() * (was / now)[:, None, :, None]).to(pool.dtype).view(torch.uint8)
        added = (rows / now[:, None, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(pool.dtype).view(torch.uint8)
        after = torch.where(is_new[..., None, None], added, torch.where(is_old[..., None, None], kept, before))
        bytes_of(pool)[0][to[:, None], :, slot] = after
        scale[0][to, :, slot[:, 0] // BLOCK] = now
    return written(s)


def plain_read(s):
    page = s["case"]["page"]
    row = torch.arange(s["rows_k"].shape[0], device="cuda")
    owner = torch.searchsorted(s["starts"][1:].long(), row, right=True)
    place = row - s["starts"].long()[owner]
    at = s["table"].long()[owner, place // page]
    s["rows_k"].copy_(block_rows(s["k"], s["k_scale"], at, place % page))
    s["rows_v"].copy_(block_rows(s["v"], s["v_scale"], at, place % page))
    return s["rows_k"], s["rows_v"]


def softmax_weights(score):
    """exp(score - max) and its sums, 1 where nothing is left (the weights are zeros then)."""
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - top.masked_fill(top == -math.inf, 0.0))
    total = weight.sum(-1, keepdim=True)
    return weight, total.masked_fill(total == 0, 1.0)


def plain_decode(s):
    case, page = s["case"], s["case"]["page"]
    n, heads, dim = case["batch"], case["heads"], case["dim"]
    cols = max(1, up(case["longest"], page))
    pages = s["table"][:, :cols].clamp(min=0).long()

    def gather(pool, scale):
        rows = bytes_of(pool)[0][pages].view(pool.dtype).float()                         # [n, cols, heads, page, D]
        rows = rows * scale[0][pages].repeat_interleave(BLOCK, dim=3)[..., None]
        return rows.transpose(1, 2).reshape(n, heads, cols * page, dim)

    live = (torch.arange(cols * page, device="cuda") < s["lengths"][:, None])[:, None, None]
    score = s["q"].float().reshape(n, heads, -1, dim) * dim ** -0.5 @ gather(s["k"], s["k_scale"]).transpose(2, 3)
    if case["bias"]:
        score[..., :case["longest"]] += s["bias"][:, None, None]
    weight, total = softmax_weights(score.masked_fill(~live, -math.inf))
    value = gather(s["v"], s["v_scale"]) * live.transpose(2, 3)
    return (weight @ value / total).reshape(n, -1, dim).to(s["q"].dtype)


def plain_cross(s):
    case, out = s["case"], torch.zeros(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    heads, dim, group = case["heads"], case["dim"], case["q_heads"] // case["heads"]
    q0 = k0 = 0
    for a, b in zip(s["queries"], s["keys"]):
        if b > 0:
            bias = s["bias"][k0:k0 + b] if case["bias"] else 0.0
            step = max(1, min(heads, (1 << 28) // (a * b * group)))                      # heads at a time: 1 GB of scores
            for h in range(0, heads, step):
                e = min(heads, h + step)
                q = s["q"][q0:q0 + a, h * group:e * group].float().reshape(a, e - h, group, dim).permute(1, 2, 0, 3).reshape(e - h, group * a, dim)
                k, v = (x[k0:k0 + b, h:e].float().transpose(0, 1) for x in (s["k"], s["v"]))
                weight, total = softmax_weights((q * dim ** -0.5) @ k.transpose(1, 2) + bias)
                got = (weight @ v / total).reshape(e - h, group, a, dim).permute(2, 0, 1, 3).reshape(a, -1, dim)
                out[q0:q0 + a, h * group:e * group] = got.to(out.dtype)
        q0, k0 = q0 + a, k0 + b
    return out


PLAIN = {"rope": plain_rope, "write": plain_write, "read": plain_read, "decode": plain_decode, "cross": plain_cross}


# ---- the same in 64 bits, from the definitions ---------------------------------------------------


def values_of(s, name, pages, count):
    """The first `count` tokens of a sequence with these pages, [heads, count, D], in 64 bits."""
    rows = [s[name][0, p].double() * s[name + "_scale"][0, p].double().repeat_interleave(BLOCK, dim=1)[..., None] for p in pages]
    return torch.cat(rows, dim=1)[:, :count]


def attention(q, k, v, bias):
    """q [h, a, D], k and v [h, b, D]."""
    score = torch.einsum("had,hbd->hab", q, k) / math.sqrt(q.shape[-1])
    if bias is not None:
        score = score + bias
    return torch.einsum("hab,hbd->had", torch.softmax(score, dim=2), v)


def exact(case, seed):
    s = prepare(case, seed)
    op, dim, heads = case["op"], case["dim"], case["heads"]
    if op == "rope":
        x, out = s["x"].double(), s["x"].double().clone()
        half = case["rotary"] // 2
        for i in range(half):
            where = s["positions"] if s["axis"] is None else s["positions"][int(s["axis"][i])]
            angle = where.double() * float(s["freqs"][i])
            turn = torch.polar(torch.ones_like(angle), -angle if case["inverse"] else angle)[:, None]
            a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
            z = torch.complex(x[..., a], x[..., b]) * turn
            out[..., a], out[..., b] = z.real, z.imag
        return out
    if op == "cross":
        if work(case)["flops"] > 2e12:
            return None
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        group = case["q_heads"] // heads
        qs, ks = s["q_starts"].tolist(), s["k_starts"].tolist()
        for b in range(case["batch"]):
            rows, keys = slice(qs[b], qs[b + 1]), slice(ks[b], ks[b + 1])
            for head in range(case["q_heads"] if ks[b + 1] > ks[b] else 0):
                out[rows, head] = attention(s["q"][rows, head].double()[None], s["k"][keys, head // group].double()[None],
                                            s["v"][keys, head // group].double()[None],
                                            s["bias"][keys].double() if case["bias"] else None)[0]
        return out
    held, add = plan(case)
    page = case["page"]
    table = [[x for x in row if x >= 0] for row in s["table"].tolist()]
    if op == "decode":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        for b, h in enumerate(held):
            if h:
                k, v = values_of(s, "k", table[b], h), values_of(s, "v", table[b], h)
                got = attention(s["q"][b].double().view(heads, -1, dim), k, v, s["bias"][b, :h].double() if case["bias"] else None)
                out[b] = got.reshape(-1, dim)
        return out
    if op == "read":
        return tuple(torch.cat([values_of(s, name, table[b], h).transpose(0, 1) for b, h in enumerate(held)]) for name in ("k", "v"))
    if s["k"].numel() > 1 << 27:
        return None
    # the pools' rows in units of their scales, and the scales
    pools = {"k": s["k"].double(), "v": s["v"].double(), "k_scale": s["k_scale"].double(), "v_scale": s["v_scale"].double()}
    refs, starts = s["refs"].tolist(), s["starts"].tolist()
    for b, h in enumerate(held):
        for _ in range(up(h + add[b], page) - up(h, page)):
            table[b].append(refs.index(0))
            refs[table[b][-1]] = 1
        for name in ("k", "v"):
            new = s["new_" + name][starts[b]:starts[b + 1]].double().transpose(0, 1)                  # [heads, tokens, D]
            if name == "v" and case["sizes"]:
                new = new + torch.log(s["sizes"][starts[b]:starts[b + 1]].double())[:, None]
            # blocks of 16: what the first one holds already, then the new rows
            front = h % BLOCK
            total = up(front + add[b], BLOCK) * BLOCK
            rows = torch.zeros((heads, total, dim), dtype=torch.float64, device="cuda")
            rows[:, front:front + add[b]] = new
            top = rows.view(heads, -1, BLOCK * dim).abs().amax(2)
            power = torch.floor(torch.log2(top.clamp(min=2.0 ** -100))) - 10
            for _ in range(3):                                       # the smallest 2^power with top <= 448 * 2^power
                power = torch.where(top > E4M3_MAX * torch.exp2(power), power + 1, power)
            scale = torch.exp2(power.clamp(LEAST, MOST))
            at = torch.tensor(table[b], device="cuda")
            place = torch.arange(h - front, h - front + total, device="cuda")
            blocks = place[::BLOCK]
            was = pools[name + "_scale"][0][at[blocks // page], :, blocks % page // BLOCK].t().clone()      # [heads, blocks]
            if front:
                scale[:, 0] = torch.maximum(scale[:, 0], was[:, 0])
                old = place[:front]
                pools[name][0][at[old // page], :, old % page] *= (was[:, 0] / scale[:, 0])[None, :, None]
            rows = (rows / scale.repeat_interleave(BLOCK, dim=1)[..., None]).clamp(-E4M3_MAX, E4M3_MAX).transpose(0, 1)
            fresh = place[front:front + add[b]]
            pools[name][0][at[fresh // page], :, fresh % page] = rows[front:front + add[b]]
            pools[name + "_scale"][0][at[blocks // page], :, blocks % page // BLOCK] = scale.t()
    return {**pools, "lengths": None, "refs": None, "table": None}
