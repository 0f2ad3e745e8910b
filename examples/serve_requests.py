"""Requests' key/value caches packed into one pool by the planner, and a serving loop over them.

A request holds a cache from the step at which it arrives until its last token, and both are known when a batch of
requests is admitted (prompt length, tokens to generate).  So its cache is a tensor of the planner: alloc_step, free_step,
and a size of whole blocks.  One greedy_by_size plan gives every request its blocks by offset -- requests that never
live together share blocks -- and the pool is as large as the plan's peak, not as the sum of the requests.

Each step writes the tokens of the requests that are in it (a prompt at a request's first step, then single tokens) and
attends over what they hold:

    python examples/serve_requests.py [--requests 48] [--check]
"""
from __future__ import annotations

import argparse
import os
import sys
from types import SimpleNamespace

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2203_00448_gb300 as mp  # noqa: E402


def requests(n, seed, prompt, generate, spread):
    """Arrival step, prompt tokens and generated tokens of n requests."""
    rng = np.random.default_rng(seed)
    return (np.sort(rng.integers(0, spread, n)), rng.integers(1, prompt + 1, n), rng.integers(1, generate + 1, n))


def plan_blocks(arrive, prompt, generate, block_tokens, device):
    """First pool block of each request, its blocks, and the pool's size, from one plan whose unit is a block."""
    blocks = -(-(prompt + generate) // block_tokens)
    n, steps = len(arrive), int((arrive + generate).max()) + 1
    trace = SimpleNamespace(trace_ptr=np.array([0, n]), steps=np.array([steps]), profile_ptr=np.array([0, steps]),
                            alloc_step=arrive, free_step=arrive + generate + 1, size_bytes=blocks, n_traces=1, max_tensors=n,
                            max_steps=steps, n_tensors=n, n_steps=steps)
    batch = mp.DeviceBatch.from_host(trace, device)
    offsets, peak, status = mp.plan_greedy_by_size(batch)
    verdict, _, _ = mp.validate_plan(batch, offsets)
    if int(status[0]) or not int(verdict[0]):
        raise RuntimeError("the requests' plan is not valid")
    return offsets.cpu().numpy(), blocks, int(peak[0])


def serve(n=48, prompt=600, generate=40, spread=60, heads=8, group=4, dim=128, block_tokens=64, seed=0, check=False,
          device="cuda", dtype=torch.bfloat16):
    """Runs the loop; returns what it did.  check: every step's outputs against plain attention over the cache read back."""
    arrive, prompts, gens = requests(n, seed, prompt, generate, spread)
    first, blocks, pool_blocks = plan_blocks(arrive, prompts, gens, block_tokens, device)
    cache = mp.KvCache(pool_blocks, block_tokens, heads, dim, device)
    held = np.zeros(n, np.int64)
    done = {"requests": n, "blocks": int(blocks.sum()), "pool_blocks": pool_blocks, "steps": 0, "tokens": 0, "worst": 0.0,
            "bytes": pool_blocks * mp.KvCache.block_bytes(block_tokens, heads, dim)}
    gen = torch.Generator(device).manual_seed(seed)
    for step in range(int((arrive + gens).max()) + 1):
        live = np.nonzero((arrive <= step) & (step <= arrive + gens))[0]
        if not len(live):
            continue
        new = np.where(held[live] == 0, prompts[live], 1)
        held[live] += new
        table = np.full((len(live), int(blocks[live].max())), -1, np.int32)
        for row, r in enumerate(live):
            table[row, :blocks[r]] = first[r] + np.arange(blocks[r])
        ptr = np.concatenate([[0], np.cumsum(new)])
        batch = mp.KvBatch(torch.from_numpy(table).to(device), torch.from_numpy(held[live].astype(np.int32)).to(device),
                           torch.from_numpy(ptr).to(device), n_tokens=int(ptr[-1]), max_tokens=int(new.max()),
                           max_len=int(held[live].max()))
        # what a layer's projection of the step's tokens leaves: queries, keys and values side by side
        qkv = torch.randn(batch.n_tokens, (group + 2) * heads * dim, device=device, generator=gen).to(dtype)
        q, k, v = (x.view(batch.n_tokens, -1, dim) for x in qkv.split([group * heads * dim, heads * dim, heads * dim], 1))
        wrote = mp.kv_write(cache, batch, k, v)
        out, _, status = mp.kv_attend(cache, batch, q)
        done["steps"] += 1
        done["tokens"] += batch.n_tokens
        if check:
            if bool(wrote.any()) or bool(status.any()):
                raise RuntimeError(f"step {step}: a sequence was refused")
            done["worst"] = max(done["worst"], difference(cache, batch, held[live], new, q, out, group))
    torch.cuda.synchronize()
    return done


def difference(cache, batch, held, new, q, out, group):
    """Largest relative (2-norm) difference of a sequence's outputs from plain attention over its cache read back."""
    everything = torch.from_numpy(np.concatenate([[0], np.cumsum(held)])).to(q.device)
    whole = mp.KvBatch(batch.table, batch.lens, everything, n_tokens=int(held.sum()))
    k, v, _ = mp.kv_read(cache, whole, dtype=torch.float32)
    worst, row, past = 0.0, 0, 0
    for length, n in zip(held, new):
        kk, vv = (x[past:past + length].repeat_interleave(group, 1).transpose(0, 1).double() for x in (k, v))
        x = q[row:row + n].transpose(0, 1).double() @ kk.transpose(1, 2) * kk.shape[-1] ** -0.5
        seen = torch.arange(length, device=q.device) <= (length - n + torch.arange(n, device=q.device))[:, None]
        want = (torch.softmax(x.masked_fill(~seen, -torch.inf), -1) @ vv).transpose(0, 1)
        worst = max(worst, float((out[row:row + n].double() - want).norm() / want.norm()))
        row, past = row + n, past + length
    return worst


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--requests", type=int, default=48)
    p.add_argument("--check", action="store_true")
    a = p.parse_args()
    d = serve(a.requests, check=a.check)
    print(f"{d['requests']} requests of {d['blocks']} blocks in all, packed into {d['pool_blocks']} "
          f"({d['bytes'] / 2**20:.1f} MiB a layer); {d['steps']} steps, {d['tokens']} tokens"
          + (f"; worst difference from plain attention {d['worst']:.2e}" if a.check else ""))
