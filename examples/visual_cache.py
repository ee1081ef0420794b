"""Compressed visual tokens in a decoder's key-value cache, end to end on one GPU.

A batch of images goes through the library the way a vision-language model uses it, with seeded random
weights in the model's place: OIM merges each image's patch tokens, the merged tokens (and a short text before and
after) enter the cache of a group of decoder layers, their values enhanced by log(size); after those layers
SPU prunes the visual tokens and the cache closes up; every image is forked into several questions; and all
questions decode, one token per step, with the step captured in a CUDA graph.

    python examples/visual_cache.py [--images 4] [--questions 3] [--steps 16] [--cache bf16|e4m3|f32]

The last step's attention is compared with dense attention over the tokens that should be in the cache, and the
largest difference printed.
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


def run(images: int = 4, questions: int = 3, steps: int = 16, cache: str = "bf16", *, side: int = 24, merged: int = 144,
        keep: int = 36, q_heads: int = 28, heads: int = 4, dim: int = 128, layers: int = 2, seed: int = 0) -> dict:
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    wide = torch.float32 if cache == "f32" else torch.bfloat16
    pool_type = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}[cache]
    width, page, before, after = q_heads * dim, 16, 9, 17

    def normal(*shape, dtype=wide):
        return torch.randn(shape, generator=g, device=dev, dtype=dtype)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=dev)

    # visual encoder -> merged tokens -> decoder width
    patches = normal(images, side, side, 256)
    tokens, sizes, _ = luvc.oim_merge(patches, merged)
    visual = tokens @ (normal(256, width) / 16)
    prompt = torch.cat((normal(images, before, width), visual, normal(images, after, width)), dim=1)
    weights = [normal(width, (q_heads + 2 * heads) * dim) / width ** 0.5 for _ in range(layers)]

    # room for the prompts, the compacted copies, and the questions' own tokens
    length = before + merged + after
    slots = images * (1 + questions)
    max_pages = -(-(length + steps) // page)
    pages = images * 2 * -(-length // page) + images * questions * (2 + -(-steps // page))
    pool = torch.zeros((layers, pages, heads, page, dim), device=dev).to(pool_type)
    scale = torch.full((layers, heads), 0.02, device=dev) if cache == "e4m3" else None
    kv = luvc.KvCache(pool, pool.clone(), slots, max_pages, k_scale=scale, v_scale=scale)

    # prompt: one ragged batch; text counts as one token, a merged token as the number it stands for
    count = torch.ones((images, length), dtype=torch.int32, device=dev)
    count[:, before:before + merged] = sizes
    luvc.kv_reserve(kv, ints([length] * images))
    starts = ints([length * i for i in range(images + 1)])
    dense = []                                                  # what each layer's cache should hold, per image
    for layer in range(layers):
        qkv = (prompt.view(-1, width) @ weights[layer]).view(-1, q_heads + 2 * heads, dim)
        k, v = qkv[:, q_heads:q_heads + heads], qkv[:, q_heads + heads:]
        luvc.kv_write(kv, k, v, layer=layer, starts=starts, sizes=count.view(-1))
        dense.append((k.view(images, length, heads, dim),
                      (v.float().view(images, length, heads, dim) + count.float().log()[..., None, None]).to(wide)))

    # after these layers the visual tokens are pruned; the cache keeps the survivors and all text
    idx, _ = luvc.spu_prune(visual, keep)
    luvc.kv_compact(kv, ints([before] * images), ints([merged] * images), idx)
    kept = torch.cat((torch.arange(before, device=dev).expand(images, -1), before + idx.long(),
                      torch.arange(before + merged, length, device=dev).expand(images, -1)), dim=1)

    # several questions about every image; the prompts' own slots are given back
    n = images * questions
    asked = torch.arange(images, dtype=torch.int32, device=dev).repeat_interleave(questions)
    slot = torch.arange(images, slots, dtype=torch.int32, device=dev)
    luvc.kv_fork(kv, asked, slot)
    luvc.kv_free(kv, torch.arange(images, dtype=torch.int32, device=dev))
    if luvc.check_status() != 0:
        raise RuntimeError("the cache reported a condition")

    # decode: room, rows and attention of every layer in one graph, page numbers worked out on the device
    one = torch.ones(n, dtype=torch.int32, device=dev)
    fresh = normal(steps, layers, n, q_heads + 2 * heads, dim)
    step_in, out = torch.empty_like(fresh[0]), torch.empty((layers, n, q_heads, dim), dtype=wide, device=dev)

    def step():
        luvc.kv_reserve(kv, one, seqs=slot)
        for layer in range(layers):
            row = step_in[layer]
            luvc.kv_write(kv, row[:, q_heads:q_heads + heads], row[:, q_heads + heads:], layer=layer, seqs=slot)
            luvc.attn_decode(row[:, :q_heads], kv, layer=layer, seqs=slot, out=out[layer])

    step_in.copy_(fresh[0])
    step()                                                      # the first step also loads the kernels
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for t in range(1, steps):
        step_in.copy_(fresh[t])
        graph.replay()
    if luvc.check_status() != 0:
        raise RuntimeError("the cache reported a condition")

    # the same attention, densely, over what should be there
    worst = 0.0
    for layer in range(layers):
        pick = kept[asked.long()]
        k, v = (torch.cat((x[asked.long()].gather(1, pick[..., None, None].expand(-1, -1, heads, dim)),
                           fresh[:, layer, :, q_heads + heads * j:q_heads + heads * (j + 1)].transpose(0, 1)), dim=1).double()
                for j, x in enumerate(dense[layer]))
        q = fresh[-1, layer, :, :q_heads].double().view(n, heads, -1, dim)
        p = torch.softmax(torch.einsum("nhgd,nthd->nhgt", q, k) * dim ** -0.5, dim=-1)
        want = torch.einsum("nhgt,nthd->nhgd", p, v).reshape(n, q_heads, dim)
        worst = max(worst, float((out[layer].double() - want).norm() / want.norm()))
    used = int((kv.refs > 0).sum())
    return {"relative_error": worst, "pages_used": used, "pages": pages, "cached_tokens": int(kv.lengths.sum()),
            "tokens_before_pruning": n * (length + steps)}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--images", type=int, default=4)
    ap.add_argument("--questions", type=int, default=3)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--cache", default="bf16", choices=["bf16", "e4m3", "f32"])
    a = ap.parse_args()
    r = run(a.images, a.questions, a.steps, a.cache)
    print("%d questions: %d tokens cached (%d without pruning), %d of %d pages in use, attention within %.2g of dense" % (
        a.images * a.questions, r["cached_tokens"], r["tokens_before_pruning"], r["pages_used"], r["pages"], r["relative_error"]))


if __name__ == "__main__":
    main()
