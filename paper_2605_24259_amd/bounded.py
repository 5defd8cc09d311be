"""A request whose live KV is bounded, beside a resident claim: the replay and the operators on the cache together.

The 60/70/80 probe (§5.3): on a pool of 80 blocks with a hard claim of 60 resident blocks an active request of 70
is refused, 60 + 70 > 80.  Bounding the active side (§3.5 mechanism table, "bound active-live KV") serves it all the
same: its prompt is taken in chunks, and after each one its cache is brought down to a budget by the attention that
its slots received, so that a chunk never needs more than what the claim leaves.  Before each chunk the replay says
whether claim, live blocks and chunk fit; without eviction it is the replay that refuses the third chunk.  Then a
tree of drafted tokens is verified over what was kept, and one token of it decoded with the account carried on.

``python -m paper_2605_24259_amd.bounded`` runs it on random keys, values and queries and prints each step.
"""
from __future__ import annotations

import math

from . import DeviceBatch, PagedCache, tracegen as tg

BLOCK = 16  # tokens
OC_ADMIT = 0


def asked(resident: int, active: int, usable: int):
    """(outcome code, blocking claim, protected blocks, required blocks) of an active request of `active` blocks beside a
    hard claim of `resident` ones."""
    trace = tg.from_pools([dict(usable_blocks=usable, mode=tg.MODE_HARD, n_chains=2, events=[
        tg.claim(resident, 0, resident, hard=1, prio=3), tg.prefill(active, 1, 0)])], "bounded")
    code, who, a, b = DeviceBatch.from_trace(trace).replay().results()[0][1].tolist()
    return code & 255, who, a, b


def run(prompt=70, chunk=10, budget=10, resident=60, usable=80, *, window=32, recent=32, heads=8, kv_heads=2, head_dim=64,
        softcap=30.0, drafts=9, evict=True, seed=0, say=lambda *a: None):
    """Blocks of `prompt` in chunks of `chunk`; the live ones brought down to `budget` after each.  Returns what
    happened: {"served" chunks, "outcomes", "length", "pos", "weight", "cache", "out", "lse", "q"...}."""
    import torch
    dev, f = "cuda", torch.bfloat16
    g = torch.Generator(device=dev).manual_seed(seed)

    def rand(*shape):
        return torch.empty(shape, device=dev).normal_(generator=g).to(f)

    def ints(*x):
        return torch.tensor(x, dtype=torch.int32, device=dev)
    blocks = usable + prompt  # of the tensors; the sequences use only what the replay admits
    k, v = rand(blocks, BLOCK, kv_heads, head_dim), rand(blocks, BLOCK, kv_heads, head_dim)
    order = torch.randperm(blocks, generator=g, device=dev).to(torch.int32)
    pages = max(resident, prompt + 1)
    table = torch.zeros(2, pages, dtype=torch.int32, device=dev)
    table[0, :resident], table[1, :prompt + 1] = order[:resident], order[resident: resident + prompt + 1]
    cache = PagedCache(k, v, table)
    held = resident * BLOCK
    n = pages * BLOCK
    weight = torch.zeros(2, kv_heads, n, device=dev)
    pos = torch.arange(n, dtype=torch.int32, device=dev).expand(2, kv_heads, n).contiguous()
    live = seen = 0  # slots of the active request, tokens of it so far
    steps, outcomes = -(-prompt // chunk), []

    def put(rows):
        """Keys and values of new tokens go behind the live slots."""
        slots = torch.arange(live, live + rows, device=dev)
        at = table[1, slots // BLOCK].long()
        k[at, slots % BLOCK], v[at, slots % BLOCK] = rand(rows, kv_heads, head_dim), rand(rows, kv_heads, head_dim)
        pos[1, :, live: live + rows] = torch.arange(seen, seen + rows, dtype=torch.int32, device=dev)

    for step in range(steps):
        rows = min(chunk, prompt - step * chunk) * BLOCK
        need = -(-(live + rows) // BLOCK)
        outcomes.append(asked(resident, need, usable))
        code, who, protected, required = outcomes[-1]
        say(f"chunk {step}: {live} live slots + {rows} tokens = {need} blocks beside {resident}: "
            + ("admitted" if code == OC_ADMIT else f"refused, claim {who}: {protected} + {required} > {usable}"))
        if code != OC_ADMIT:
            return dict(served=step, outcomes=outcomes, length=live, cache=cache)
        put(rows)
        q = rand(rows, heads, head_dim) * 3
        length, offset = ints(held, live + rows), ints(0, 0, rows)
        out, lse = cache.attend(q, offset, length, max_rows=rows, max_len=n, softcap=softcap)
        # the account goes by the chunk's last rows
        w = min(window, rows)
        weight[1, :, live: live + rows] = 0
        weight = cache.weigh(q[-w:], lse[-w:].contiguous(), ints(0, 0, w), length, max_rows=w, max_len=n, softcap=softcap,
                             weight=weight)
        live, seen = live + rows, seen + rows
        if evict and live > budget * BLOCK:
            length, weight, pos = cache.evict(weight, length, ints(held, budget * BLOCK), protect=ints(held, BLOCK),
                                              recent_from=ints(1 << 30, seen - recent), pos=pos)
            live = budget * BLOCK  # min(length, max(budget, protect))
            say(f"         {rows} rows attended, {live} slots kept")

    # drafted tokens: a root that continues the prompt, and children of earlier ones
    parent = torch.tensor([-1] + [i // 2 for i in range(drafts - 1)], dtype=torch.int32, device=dev)
    put(drafts)
    q = rand(drafts, heads, head_dim) * 3
    offset, length = ints(0, 0, drafts), ints(held, live + drafts)
    out, lse = cache.attend(q, offset, length, max_rows=drafts, max_len=n, softcap=softcap, parent=parent)
    drafted = dict(q=q, out=out, lse=lse, parent=parent, length=live + drafts)
    # the root was accepted: decode it with the account carried on
    weight[1, :, live: live + 1] = 0
    length = ints(held, live + 1)
    out, lse, weight = cache.attend(q[:1], ints(0, 0, 1), length, max_rows=1, max_len=n, softcap=softcap, weight=weight, decay=0.99)
    say(f"tree of {drafts} drafted tokens verified, one token decoded over {live + 1} slots of {seen + 1} tokens")
    return dict(served=steps, outcomes=outcomes, length=live + 1, pos=pos, weight=weight, cache=cache, q=q[:1], out=out,
                lse=lse, drafted=drafted, scale=1 / math.sqrt(head_dim), softcap=softcap, held=held, tokens=seen + 1)


def main():
    print("whole: outcome %d (claim %d: protected %d, required %d, usable 80)" % asked(60, 70, 80))
    for evict in (False, True):
        print("with eviction" if evict else "without eviction")
        r = run(evict=evict, say=lambda *a: print("  ", *a))
        print(f"   {r['served']} chunks served")
    if r["cache"].status.any().item():
        raise RuntimeError("the cache's status words are not zero")


if __name__ == "__main__":
    main()
