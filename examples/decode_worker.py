#!/usr/bin/env python3
"""A decode worker on one GPU: a request's KV arrives as payloads (kvc_compress on the prefill side), is rebuilt once, and from then
on lives in pages of codes.  Every step writes a tree of drafted tokens, attends it over the pages, keeps an accepted path and
goes on; at the end the KV, with the new tokens, is read back and compressed for the next movement.

The model around it is left out: queries, keys and values of the drafts are random, and the accepted path is the one whose
last token's query agrees most with its output.  Run: python examples/decode_worker.py [--prompt 1000 --steps 8 --drafts 16]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_13734_amd import kvc, kvgen  # noqa: E402

DIM = 128


def draft_tree(n, g):
    """Parents of n drafts (-1: the last accepted token) and, per draft, the bits of its ancestors and itself."""
    parent, bits = [], []
    for i in range(n):
        p = int(torch.randint(max(-1, i - 4), i, (1,), generator=g)) if i else -1
        parent.append(p)
        bits.append((1 << i) | (bits[p] if p >= 0 else 0))
    return parent, [b - (1 << 64) if b >> 63 else b for b in bits]


def path_to(parent, node):
    path = []
    while node >= 0:
        path.append(node)
        node = parent[node]
    return path[::-1]


def run(prompt=1000, steps=8, drafts=16, layers=2, kv_heads=8, q_heads=32, seed=0, device="cuda"):
    """Returns (tokens in the cache, their K and V as the cache holds them, the last layer's last step: (q, k, v, out of
    the drafts, tokens before them))."""
    assert 1 <= drafts <= 64
    stream = torch.cuda.current_stream().cuda_stream
    g = torch.Generator().manual_seed(seed)
    gd = torch.Generator(device=device).manual_seed(seed)
    most = prompt + steps * drafts

    # ---- the movement: one payload for all layers, rebuilt at the receiver
    x = kvgen.make_kv(seed, layers, kv_heads, DIM, prompt, torch.float16, device)
    plan = kvc.Plan(kvc.F16, layers, kv_heads, DIM, 8, 4, 64, 64, max_tokens=most, transform=1)
    wire = kvc.Buffers(plan, [prompt], device)
    wire.compress([kvc.contiguous_request(x)], stream)
    rebuilt = torch.empty_like(x)
    wire.decompress([kvc.contiguous_request(rebuilt)], stream)

    # ---- the cache: pages of 32 tokens, one pool per layer, one block table for all; K rotated, since its channels differ in size
    cache_plan = kvc.CachePlan(kvc.F16, kv_heads, q_heads, DIM, 8, 4, 64, 32, kvc.T_HADAMARD, max_tokens=most, max_new=drafts)
    pages = (most + 31) // 32
    caches = []
    for _ in range(layers):
        caches.append(kvc.Cache(cache_plan, pages, device, caches[0].workspace if caches else None))
    table = torch.randperm(pages, generator=g).to(torch.int32).reshape(1, -1).to(device)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=device)                     # noqa: E731
    tokens = prompt
    prompt_rows = kvc.CacheBatch(i32(0, prompt), i32(tokens), table, prompt, most, pages)
    for l, cache in enumerate(caches):                   # (rows by their strides: nothing is transposed in memory)
        cache.store(prompt_rows, rebuilt[l, 0].transpose(0, 1), rebuilt[l, 1].transpose(0, 1), stream)

    # ---- steps
    scale = DIM ** -0.5
    last = None
    for _ in range(steps):
        parent, bits = draft_tree(drafts, g)
        mask = torch.tensor(bits, dtype=torch.int64, device=device).reshape(-1, 1)
        batch = kvc.CacheBatch(i32(0, drafts), i32(tokens + drafts), table, drafts, most, pages, mask)
        score = torch.zeros(drafts, device=device)
        for cache in caches:
            k, v = (torch.randn(drafts, kv_heads, DIM, generator=gd, device=device).half() for _ in range(2))
            q = torch.randn(drafts, q_heads, DIM, generator=gd, device=device).half()
            out = torch.empty_like(q)
            cache.store(batch, k, v, stream)
            cache.attend(batch, q, out, scale, stream=stream)
            score += (q.float() * out.float()).sum((1, 2))
            last = (q, k, v, out, tokens)
        path = path_to(parent, int(score.argmax()))      # the step's one look at the GPU
        keep_start, keep = i32(0, len(path)), i32(*path)
        for cache in caches:
            cache.keep(batch, keep_start, keep, stream)
        tokens += len(path)

    # ---- the next movement: everything read back, layer by layer, into the layout of a request, and compressed
    back = torch.empty(layers, 2, kv_heads, tokens, DIM, dtype=torch.float16, device=device)
    everything = kvc.CacheBatch(i32(0, tokens), i32(tokens), table, tokens, most, pages)
    for l, cache in enumerate(caches):
        cache.load(everything, back[l, 0].transpose(0, 1), back[l, 1].transpose(0, 1), stream)
    out_wire = kvc.Buffers(plan, [tokens], device)
    out_wire.compress([kvc.contiguous_request(back)], stream)
    torch.cuda.synchronize()
    for status in [wire.status, out_wire.status] + [c.status for c in caches]:
        assert not status.any(), status
    held = sum(c.pages.numel() for c in caches)
    print("%d prompt tokens + %d accepted of %d drafted; cache %.2f MB (%.2f MB at 16 bits), next payload %.2f MB" % (
        prompt, tokens - prompt, steps * drafts, held / 1e6, pages * 32 * layers * kv_heads * DIM * 4 / 1e6, int(out_wire.out_bytes[0]) / 1e6))
    return tokens, back, last


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    for name, default in (("prompt", 1000), ("steps", 8), ("drafts", 16), ("layers", 2)):
        ap.add_argument("--" + name, type=int, default=default)
    run(**vars(ap.parse_args()))
