"""The time of a recomputed token, measured: the requests of a trace served from
a paged KV cache on the GPU.

The objectives charge every token that no tier holds ``t_prefill_per_token``
seconds (kv_cost_model).  Kareto takes such times from profiles of the target GPU
(Section 3.2); this module takes the part that a cache decides on, attention and
the cache's own upkeep, from the card itself.  A trace's requests run in
batches over a cache of fixed-size blocks in HBM: a request reuses the blocks of
its prefix that are cached, brings the rest as new tokens, and the blocks used
longest ago make room.  Every batch is one serving step of the operators in
:mod:`.kvpaged`: plan, then for a layer rotation and cache write, then attention.

    python -m paper_2603_08739_amd.prefill_cost --requests 256 --layers 32

prints what was measured and the objectives of a small grid under it.
"""
from __future__ import annotations

import argparse
import collections
import itertools
import json

import numpy as np
import torch

from . import kvpaged


class BlockPool:
    """Blocks of an HBM cache by the hash of what they hold; the least recently used
    unpinned ones are given away when none is free."""

    def __init__(self, n_blocks):
        self.free = collections.deque(range(n_blocks))
        self.held = collections.OrderedDict()  # hash -> block, oldest use first

    def prefix(self, hashes):
        """Blocks of the cached run at the front of `hashes`, now used."""
        run = []
        for h in hashes:
            if h not in self.held:
                break
            self.held.move_to_end(h)
            run.append(self.held[h])
        return run

    def take(self, n, pinned):
        """n blocks for new contents; none of `pinned` (hashes) is given away.  None, and
        nothing is given away, if there are not so many."""
        old = max(0, n - len(self.free))
        if old > len(self.held) - sum(h in self.held for h in pinned):
            return None
        out = [self.free.popleft() for _ in range(n - old)]
        oldest = itertools.islice((h for h in self.held if h not in pinned), old)
        return out + [self.held.pop(h) for h in list(oldest)]

    def keep(self, h, block):
        """`block` holds h from now on; given back if another block does already."""
        if h in self.held:
            self.free.append(block)
        else:
            self.held[h] = block


def requests_of(trace):
    """Per request, the list of its block hashes."""
    cuts = np.flatnonzero(np.diff(trace.req)) + 1
    return [part.tolist() for part in np.split(trace.hash, cuts)]


def batches(trace, n_blocks, batch):
    """Serving steps: (cached blocks, blocks taken) of every request of a batch.  A
    request whose blocks are all cached computes its last one again: an answer
    needs a token.  One that does not fit the cache, or with which the step would bring
    more new tokens than a plan takes, ends the batch; alone, it is skipped."""
    pool, waiting = BlockPool(n_blocks), collections.deque(requests_of(trace))
    block = trace.tokens_per_granule * (int(trace.weight.max()) if len(trace.weight) else 1)
    while waiting:
        step, pinned, fresh = [], set(), []
        room = kvpaged.KV_PAGED_MAX_TOKENS // block  # new blocks that the step may still bring
        while waiting and len(step) < batch:
            hashes = waiting[0]
            run = pool.prefix(hashes)[:len(hashes) - 1]
            new = len(hashes) - len(run)
            got = pool.take(new, pinned | set(hashes[:len(run)])) if new <= room else None
            if got is None:
                if not step:
                    waiting.popleft()
                break
            waiting.popleft()
            room -= new
            pinned |= set(hashes[:len(run)])
            step.append((run, got))
            fresh += list(zip(hashes[len(run):], got))
        for h, block_of in fresh:
            pool.keep(h, block_of)
        if step:
            yield step


def measure(trace, n_blocks, batch=16, max_requests=None, q_heads=32, kv_heads=8, head_dim=128, dtype=torch.bfloat16,
            base=500000.0, seed=0, device="cuda"):
    """Runs the trace's first requests; one layer's seconds and token counts."""
    weights = np.unique(trace.weight)
    if len(weights) != 1:
        raise ValueError("the requests' blocks must have one size")
    if max_requests is not None and max_requests < 1:
        raise ValueError("max_requests must be at least 1")
    block = int(trace.tokens_per_granule * weights[0])
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    k = torch.zeros(n_blocks, kv_heads, block, head_dim, dtype=dtype, device=device)
    v = torch.zeros(n_blocks, kv_heads, head_dim, block, dtype=dtype, device=device)
    cache, rope = kvpaged.Cache(k, v), kvpaged.Rope(head_dim, base=base)
    i32 = dict(dtype=torch.int32, device=device)
    done = dict(requests=0, steps=0, cached_tokens=0, new_tokens=0, plan_s=0.0, append_s=0.0, attention_s=0.0)

    def serve(step):  # one step's tensors are let go before the next one's are made
        ctx = [len(run) * block for run, _ in step]
        new = [len(got) * block for _, got in step]
        columns = max(len(run) + len(got) for run, got in step)
        rows = [run + [-1] * (columns - len(run)) for run, _ in step]
        table, free = torch.tensor(rows, **i32), torch.tensor([b for _, got in step for b in got], **i32)
        lens = torch.tensor(ctx, **i32), torch.tensor(new, **i32)
        total = sum(new)
        fused = torch.randn(total, q_heads + 2 * kv_heads, head_dim, generator=g, device=device, dtype=dtype)
        q = fused[:, :q_heads]
        out = torch.empty(total, q_heads, head_dim, device=device, dtype=dtype)
        plan = kvpaged.Plan(len(step), total, block, columns, q_heads, kv_heads, head_dim, max_new=max(new), device=device)
        for warm in (True, False):  # a first step of new sizes is not the one that counts
            at = [torch.cuda.Event(enable_timing=True) for _ in range(4)]
            at[0].record()
            kvpaged.kv_paged_plan(plan, *lens, table, free)
            at[1].record()
            kvpaged.kv_paged_append(plan, cache, fused[:, q_heads:q_heads + kv_heads], fused[:, q_heads + kv_heads:],
                                    q=q, q_out=q if not warm else out, rope=rope)
            at[2].record()
            kvpaged.kv_paged_attention(plan, cache, q, out=out)
            at[3].record()
        done["requests"] += len(step)
        done["steps"] += 1
        done["cached_tokens"] += sum(ctx)
        done["new_tokens"] += total
        return at, plan.result  # not the plan: its work memory is tens of megabytes

    marks = []
    for step in batches(trace, n_blocks, batch):
        if max_requests is not None:
            step = step[:max_requests - done["requests"]]
        marks.append(serve(step))
        if max_requests is not None and done["requests"] >= max_requests:
            break
    torch.cuda.synchronize()
    for at, result in marks:
        if result[3].item():
            raise RuntimeError(f"a step's plan was refused: {result.tolist()}")
        for i, name in enumerate(("plan_s", "append_s", "attention_s")):
            done[name] += at[i].elapsed_time(at[i + 1]) * 1e-3
    rope.free()
    return done


def seconds_per_token(done, layers, other=0.0):
    """t_prefill_per_token of a model of so many layers; `other`: seconds a token spends
    outside attention and cache (the products with the weights)."""
    if not done["new_tokens"]:
        raise ValueError("nothing was recomputed")
    return (done["plan_s"] + layers * (done["append_s"] + done["attention_s"])) / done["new_tokens"] + other


def main(argv=None):
    import tracegen as tg
    from . import host
    ap = argparse.ArgumentParser(description="measure t_prefill_per_token on this GPU and evaluate a grid under it")
    ap.add_argument("--requests", type=int, default=256)
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--blocks", type=int, default=16384, help="blocks of the HBM cache")
    ap.add_argument("--layers", type=int, default=32)
    ap.add_argument("--other-us", type=float, default=0.0, help="microseconds a token spends in the products with the weights")
    a = ap.parse_args(argv)
    trace = tg.tiny(n_req=max(a.requests, 1))
    done = measure(trace, a.blocks, batch=a.batch, max_requests=a.requests)
    t = seconds_per_token(done, a.layers, a.other_us * 1e-6)
    cfgs = tg.configs_for("tiny", trace)
    handle = host.load(trace)
    _, obj = host.evaluate(handle, cfgs, dict(tg.DEFAULT_COST, t_prefill_per_token=t), trace.n_groups)
    handle.free()
    flags, n = host.pareto(obj)
    holds = "attention and the cache's upkeep, measured; " + (
        "the products with the weights as given by --other-us" if a.other_us else "without the products with the weights (--other-us)")
    print(json.dumps({**{k: round(v, 6) for k, v in done.items()}, "layers": a.layers, "other_s_per_token": a.other_us * 1e-6,
                      "t_prefill_per_token": t, "t_prefill_per_token_holds": holds, "configs": int(cfgs.n), "front": int(n)}))
    return done, t, obj, flags


if __name__ == "__main__":
    main()
