"""Questions about merged images, end to end on one GPU: positions, an 8-bit cache, and the attention to the images' tokens.

With seeded random weights in a model's place: OIM merges each image's patch tokens; a merged token stands at the mean row and column
of its patches, and its key is turned by them (luvc.rope, frame, row and column each for its own frequencies); keys and values, enhanced
by log(size), are quantised into a paged cache with a scale for each 16 tokens of a head; the rows are read back as the states that the
tokens of each question look at (luvc.attn_cross); and one more token of each question decodes over the same cache.  A merged token's size
counts once, in its values; with values as they are it would be the key_bias of both calls instead.

    python examples/visual_question.py [--images 4] [--tokens 23] [--heads 28]

Both results are compared with dense attention over the rows that the cache stands for, and the largest differences printed.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2512_09010_b200 as luvc  # noqa: E402


def run(images: int = 4, tokens: int = 23, q_heads: int = 28, *, side: int = 24, merged: int = 144, heads: int = 4, dim: int = 128,
        seed: int = 0) -> dict:
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    width, page = q_heads * dim, 16

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.bfloat16)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=dev)

    # visual encoder -> merged tokens; where their patches were, on average
    patches = normal(images, side, side, 256)
    visual, sizes, owner = luvc.oim_merge(patches, merged)
    place = torch.arange(side * side, device=dev).expand(images, -1)
    where = torch.zeros((2, images, merged), device=dev)
    for axis, x in enumerate((place // side, place % side)):
        where[axis].scatter_add_(1, owner.long(), x.float())
    where = (where / sizes).round().int()
    frame = torch.zeros_like(where[:1])
    positions = torch.cat((frame, where)).view(3, -1).contiguous()              # of all merged tokens: (frame, row, column)

    # a quarter of the frequencies for the frame, three eighths each for row and column
    freqs, factor = luvc.rope_frequencies(dim, device=dev)
    axis = ints([0] * (dim // 8) + [1] * (3 * dim // 16) + [2] * (3 * dim // 16))
    weight = normal(256, 2 * heads * dim) / 16
    kv = (visual.reshape(-1, 256) @ weight).view(-1, 2 * heads, dim)
    k, v = kv[:, :heads], kv[:, heads:]
    luvc.rope(k, positions, freqs, axis=axis, factor=factor, out=k)             # in place, beside the values

    # the cache
    cols = -(-merged // page)
    pool = torch.zeros((1, images * cols, heads, page, dim), device=dev).to(torch.float8_e4m3fn)
    scale = torch.zeros((1, images * cols, heads, page // luvc.KV_BLOCK), device=dev)
    cache = luvc.KvCache(pool, pool.clone(), images, cols, k_scale=scale, v_scale=scale.clone())
    starts = ints([merged * i for i in range(images + 1)])
    luvc.kv_reserve(cache, ints([merged] * images))
    luvc.kv_write(cache, k, v, starts=starts, sizes=sizes.view(-1))

    # the questions' tokens look at the images: all heads of a token at once, without an order among the states
    text = normal(images * tokens, width) @ (normal(width, width) / width ** 0.5)
    q = text.view(-1, q_heads, dim)
    asked = ints([side + i for i in range(tokens)] * images)                    # behind the image
    q = luvc.rope(q, asked.expand(3, -1), freqs, axis=axis, factor=factor)
    states = torch.empty_like(kv)
    luvc.kv_read(cache, states[:, :heads], states[:, heads:], starts=starts)
    seen = luvc.attn_cross(q, states[:, :heads], states[:, heads:], q_starts=ints([tokens * i for i in range(images + 1)]), k_starts=starts)
    # one more token of each decodes over the cache as it is
    last = q.view(images, tokens, q_heads, dim)[:, -1]
    answer = luvc.attn_decode(last, cache)
    if luvc.check_status() != 0:
        raise RuntimeError("a call reported a condition")

    # the same, densely
    ks, vs = (states.view(images, merged, 2, heads, dim)[:, :, j].double() for j in (0, 1))
    score = torch.einsum("nthgd,nshd->nhgts", q.double().view(images, tokens, heads, -1, dim), ks) * dim ** -0.5
    p = torch.softmax(score, dim=-1)
    want = torch.einsum("nhgts,nshd->nthgd", p, vs).reshape(images, tokens, q_heads, dim)
    exact = v.double() + sizes.view(-1).double().log()[:, None, None]
    return {"cross_error": float((seen.double().view_as(want) - want).norm() / want.norm()),
            "decode_error": float((answer.double() - want[:, -1]).norm() / want[:, -1].norm()),
            "cache_error": float((states[:, heads:].double() - exact).norm() / exact.norm()),
            "cached_tokens": int(cache.lengths.sum())}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--images", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=23)
    ap.add_argument("--heads", type=int, default=28)
    a = ap.parse_args()
    r = run(a.images, a.tokens, a.heads)
    print("%d tokens cached, values within %.2g of the projection's; questions within %.2g of dense attention, decoded tokens within %.2g" % (
        r["cached_tokens"], r["cache_error"], r["cross_error"], r["decode_error"]))


if __name__ == "__main__":
    main()
