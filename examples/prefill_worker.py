#!/usr/bin/env python3
"""A prefill worker on one GPU: requests of different lengths arrive together, their queries and keys are normed per head and rotated, the
prompts are attended in 16 bits, K and V go into pages of codes and, for the first request, into a payload for a decode worker
elsewhere.  Then the worker decodes some tokens of all requests itself, and the requests end one after the other.

The lengths, block tables, positions and free pages live on the GPU (kvc_cache_advance): the host knows the prompts' lengths, nothing else.
The model around it is left out: projections are random.  Run: python examples/prefill_worker.py [--steps 4]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_13734_amd import kvc  # noqa: E402

DIM = 128


def run(lengths=(900, 37, 411), steps=4, layers=2, kv_heads=8, q_heads=32, seed=0, device="cuda"):
    """Returns the last layer's (rotated q, k, v, out of the prompts, starts), and of every step (rotated q, k, v, out); all per row."""
    stream = torch.cuda.current_stream().cuda_stream
    g = torch.Generator(device=device).manual_seed(seed)
    n, rows, most = len(lengths), sum(lengths), max(lengths) + steps
    scale = DIM ** -0.5
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=device)                     # noqa: E731

    def heads(rows):
        """What a layer's projection leaves: queries, keys and values of all rows, in one tensor."""
        x = torch.randn(rows, q_heads + 2 * kv_heads, DIM, generator=g, device=device).half()
        return x[:, :q_heads], x[:, q_heads: q_heads + kv_heads], x[:, q_heads + kv_heads:]

    # ---- plans, one set of tables and a pool of pages per layer
    frequencies = kvc.rotary_frequencies(DIM, 500000.0, kvc.SCALE_BANDS, 8.0, 1.0, 4.0, 8192)
    prompt = kvc.Prompt(kvc.PromptPlan(kvc.F16, kv_heads, q_heads, frequencies=frequencies, eps=1e-6, max_batch=n), device)
    weights = [(1 + 0.1 * torch.randn(DIM, generator=g, device=device)).half() for _ in "qk"]
    cache_plan = kvc.CachePlan(kvc.F16, kv_heads, q_heads, DIM, 8, 8, 64, 32, kvc.T_HADAMARD, max_batch=n, max_tokens=most)
    num_pages = sum((t + steps + 31) // 32 for t in lengths)
    pages = kvc.CachePages(cache_plan, num_pages, n, device)
    caches = []
    for _ in range(layers):
        caches.append(kvc.Cache(cache_plan, num_pages, device, caches[0].workspace if caches else None))
    start, tokens, positions = i32(*[0] * (n + 1)), i32(*[0] * n), i32(*[0] * rows)

    # ---- the prompts: where their tokens are and go, then layer by layer
    pages.advance(start, tokens, fresh=i32(*lengths), max_new=max(lengths), positions=positions, stream=stream)
    batch, new = kvc.PromptBatch(start, max(lengths)), kvc.CacheBatch(start, tokens, pages.table, max(lengths), most, num_pages)
    sent = torch.empty(layers, 2, kv_heads, lengths[0], DIM, dtype=torch.float16, device=device)
    for l, cache in enumerate(caches):
        q, k, v = heads(rows)
        prompt.rotate(q, k, positions, q_weight=weights[0], k_weight=weights[1], stream=stream)
        out = torch.empty(rows, q_heads, DIM, dtype=torch.float16, device=device)
        prompt.attend(batch, q, k, v, out, scale, stream=stream)
        cache.store(new, k, v, stream)
        for x, to in zip((k, v), sent[l]):
            to.copy_(x[: lengths[0]].transpose(0, 1))
    prompts = (q, k, v, out, start.tolist())

    # ---- the first request's movement
    plan = kvc.Plan(kvc.F16, layers, kv_heads, DIM, 4, 4, 32, 32, codec=kvc.CODEC_HUFF8, max_tokens=lengths[0])
    wire = kvc.Buffers(plan, [lengths[0]], device)
    wire.compress([kvc.contiguous_request(sent)], stream)

    # ---- steps of one token per request
    one, positions = i32(*[1] * n), i32(*[0] * n)
    step = kvc.CacheBatch(start, tokens, pages.table, 1, most, num_pages)
    done = []
    for _ in range(steps):
        pages.advance(start, tokens, fresh=one, max_new=1, positions=positions, stream=stream)
        for cache in caches:
            q, k, v = heads(n)
            prompt.rotate(q, k, positions, q_weight=weights[0], k_weight=weights[1], stream=stream)
            out = torch.empty(n, q_heads, DIM, dtype=torch.float16, device=device)
            cache.store(step, k, v, stream)
            cache.attend(step, q, out, scale, stream=stream)
        done.append((q, k, v, out))

    # ---- the requests end, and their pages are free again
    torch.cuda.synchronize()
    used = num_pages - int(pages.free_count)
    for i in range(n):
        pages.advance(start, tokens, kept=torch.where(torch.arange(n, device=device) <= i, 0, pages.held).int(), stream=stream)
    torch.cuda.synchronize()
    for status in [wire.status, pages.status, prompt.status] + [c.status for c in caches]:
        assert not status.any(), status
    assert int(pages.free_count) == num_pages and not pages.held.any()
    print("%d prompts, %d tokens, %d steps; %d pages in use, payload of the first %.2f MB of %.2f" % (
        n, rows, steps, used, int(wire.out_bytes[0]) / 1e6, sent.numel() * 2 / 1e6))
    return prompts, done


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=4)
    run(**vars(ap.parse_args()))
