"""Generation over compressed prompts in a paged 4-bit cache: one layer of a few requests, with random weights and inputs.

  1. prefill_compress keeps whole shots of each prompt under a token budget (a different number of rows per request);
  2. pages_plan takes pages for the kept rows, store puts them there in 4 bits, and the bf16 rows can go;
  3. every step, pages_plan finds the new tokens' places, qk_norm_rope normalises and rotates their queries and keys and
     stores keys and values, attention runs over kept and generated tokens;
  4. pages_release gives everything back.

Keys of the prompt are taken as rotated already, as they would be when the prompt was processed.  Run from the repository's
root: python examples/paged_generation.py [--steps 64] [--requests 8]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2502_01941_amd import kv4, shotkv, workloads as wl  # noqa: E402

PAGE = 64


def rotation(positions, dim, base=500000.0):
    """Table of kv4.Rope: cosines and sines of every position's dim / 2 angles."""
    pair = torch.arange(dim // 2, dtype=torch.float64, device="cuda")
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * base ** (-2 * pair / dim)
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def generate(requests=8, steps=64, prompt=4096, shots=20, budget=1024, q_heads=32, kv_heads=8, head_dim=128, seed=0):
    """Runs the loop; returns what a check needs."""
    shape = wl.PrefillShape("paged", requests, q_heads, kv_heads, head_dim, 32, prompt, shots, torch.bfloat16, budget)
    q, k, v, offsets, budgets = wl.prefill_batch(shape, "cuda", seed)
    kept = shotkv.prefill_compress(q, k, v, offsets, budgets, budget, shape.sm_scale)

    # a pool of pages for all that may come, a block table, the stack of free pages
    per_request = -(-(budget + steps) // PAGE)
    cache = kv4.Cache.empty(requests * per_request, PAGE, kv_heads, head_dim)
    table = torch.full((requests, per_request), -1, dtype=torch.int32, device="cuda")
    free = torch.arange(cache.n_pages, dtype=torch.int32, device="cuda")
    count = torch.full((1,), cache.n_pages, dtype=torch.int32, device="cuda")
    lens = torch.zeros(requests, dtype=torch.int32, device="cuda")

    # the kept rows of every request, a batch of equal shares of `budget` tokens
    plan = kv4.PagePlan.empty(table, requests * budget)
    kv4.pages_plan(PAGE, lens, kept.kept_count, free, count, plan, request_tokens=budget)
    kv4.store(cache, kept.k_out.transpose(1, 2), kept.v_out.transpose(1, 2), plan.slot_map)
    lens.copy_(plan.seq_lens)
    count.copy_(plan.free_left)
    in_cache = lens.clone()
    kept.k_out = kept.v_out = None

    # generation: one new token per request and step
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    weight = [(1 + 0.1 * torch.randn(head_dim, generator=gen, device="cuda")).bfloat16() for _ in range(2)]
    rope = kv4.Rope(rotation(prompt + steps, head_dim), weight[0], weight[1])
    step_plan = kv4.PagePlan.empty(table, requests)
    one = torch.ones(requests, dtype=torch.int32, device="cuda")
    position = torch.full((requests,), prompt, dtype=torch.int32, device="cuda")    # of the next token, not its place in the cache
    rotated = torch.empty((requests, q_heads, head_dim), dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(rotated)
    workspace = kv4.attention_workspace(cache, rotated, table)
    for _ in range(steps):
        qkv = torch.randn((requests, q_heads + 2 * kv_heads, head_dim), generator=gen, device="cuda").bfloat16()
        kv4.pages_plan(PAGE, lens, one, free, count, step_plan, position)
        kv4.qk_norm_rope(rope, qkv[:, :q_heads], qkv[:, q_heads:q_heads + kv_heads], step_plan.token_pos, rotated, None,
                         qkv[:, q_heads + kv_heads:], cache, step_plan.slot_map)
        lens.copy_(step_plan.seq_lens)
        count.copy_(step_plan.free_left)
        position += 1
        kv4.attention(cache, rotated, table, lens, shape.sm_scale, out=out, workspace=workspace)
    last = {"q": rotated, "out": out, "lens": lens.clone(), "in_cache": in_cache, "table": table.clone(), "cache": cache,
            "scale": shape.sm_scale, "status": step_plan.status}
    kv4.pages_release(PAGE, torch.ones(requests, dtype=torch.uint8, device="cuda"), lens, table, free, count)
    last.update(left=count, free=free)
    return last


def main():
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--requests", type=int, default=8)
    parser.add_argument("--steps", type=int, default=64)
    args = parser.parse_args()
    last = generate(args.requests, args.steps)
    torch.cuda.synchronize()
    cache, tokens = last["cache"], int(last["lens"].sum())
    print(f"{args.requests} requests, {args.steps} steps: {tokens} tokens in the cache, "
          f"{last['in_cache'].tolist()} of them kept of the prompts")
    print(f"{cache.pages.numel() / tokens / cache.n_kv_heads:.1f} bytes of pages per token and KV head "
          f"({cache.head_dim * 17 // 16} of codes and scales; bf16 rows have {cache.head_dim * 4})")
    print(f"pages back on the stack: {int(last['left'])} of {cache.n_pages}")


if __name__ == "__main__":
    main()
