"""Plain implementation of the operators on a paged KV cache, in 64 bits on the CPU, row by row."""
from __future__ import annotations

import math

import numpy as np


class Case:
    """A cache, its sequences and the rows of a call, on the CPU; values from a seed."""

    def __init__(self, seed, lens, rows, *, kv_heads=2, group=3, dim=64, dtype="bfloat16", page=16, softcap=0.0, bias=False,
                 parent=None, row_start=None, prefix=None, scale=None, layout="slots first", gap=0):
        import torch
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.lens, self.rows, self.page, self.dim = list(lens), list(rows), page, dim
        self.kv_heads, self.group, self.softcap = kv_heads, group, softcap
        self.scale = 1 / math.sqrt(dim) if scale is None else scale
        self.dtype = getattr(torch, dtype)
        S, pages = len(self.lens), max(1, -(-max(self.lens, default=1) // page)) + 1
        blocks = S * pages + 2
        shape = {"slots first": (blocks, page, kv_heads, dim), "heads first": (blocks, kv_heads, page, dim)}[layout]
        wide = shape[:3] + (dim + gap,)
        self.k, self.v = (torch.randn(wide, generator=g).to(self.dtype)[..., :dim] for _ in range(2))
        if layout == "heads first":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.table = torch.from_numpy(rng.permutation(blocks)[: S * pages].reshape(S, pages).astype(np.int32))
        T, Q = sum(self.rows), kv_heads * group
        self.q = (torch.randn(T, Q, dim, generator=g) * (8 if softcap else 2)).to(self.dtype)
        self.offset = np.concatenate([[0], np.cumsum(self.rows)]).astype(np.int32)
        self.slope = torch.rand(Q, generator=g) * 0.3 if bias else None
        self.parent, self.row_start, self.prefix = parent, row_start, prefix
        self.weight = torch.rand(S, kv_heads, max(self.lens, default=0) + 3, generator=g)
        # behind the lengths, in the table's spare pages and in blocks of nobody: anything
        for s, n in enumerate(self.lens):
            for j in range(n, pages * page):
                self.k[self.table[s, j // page], j % page] = float("nan")
                self.v[self.table[s, j // page], j % page] = float("nan") if j % 2 else float("inf")

    def slots(self, pool, s, h):
        return np.stack([pool[self.table[s, j // self.page], j % self.page, h].double().numpy() for j in range(self.lens[s])]) \
            if self.lens[s] else np.zeros((0, self.dim))

    def seen(self, s):
        """(see [rows, len], distance [rows, len]) of a sequence."""
        n, r, o = self.lens[s], self.rows[s], int(self.offset[s])
        base, j = n - r, np.arange(n)
        see, pos, place = np.zeros((r, n), bool), np.zeros(r, int), np.arange(n)
        pre = 0 if self.prefix is None else max(0, min(self.prefix[s], n if self.parent is None else base))
        lines = []
        for i in range(r):
            start = 0 if self.row_start is None else self.row_start[o + i]
            if self.parent is None:
                see[i] = (j >= start) & (j <= base + i)
                pos[i] = base + i
            else:
                p = self.parent[o + i]
                lines.append((lines[p] if p >= 0 else []) + [i])
                see[i] = (j >= start) & (j < base)
                see[i, [base + a for a in lines[i]]] = True
                pos[i] = place[base + i] = base + len(lines[i]) - 1
            see[i, :pre] = True
        return see, np.abs(pos[:, None] - place[None])

    def scores(self, s, head):
        x = self.q[self.offset[s]: self.offset[s + 1], head].double().numpy() @ self.slots(self.k, s, head // self.group).T
        x = x * self.scale
        if self.softcap:
            x = self.softcap * np.tanh(x / self.softcap)
        see, far = self.seen(s)
        if self.slope is not None:
            x = x - float(self.slope[head]) * far
        return x, see

    def attend(self):
        T, Q = self.q.shape[:2]
        out, lse = np.zeros((T, Q, self.dim)), np.full((T, Q), -np.inf)
        for s in range(len(self.lens)):
            for head in range(Q):
                x, see = self.scores(s, head)
                v = self.slots(self.v, s, head // self.group)
                for i in range(self.rows[s]):
                    t, at = int(self.offset[s]) + i, np.nonzero(see[i])[0]
                    if not at.size:
                        continue
                    with np.errstate(all="ignore"):
                        y = x[i, at]
                        m = y.max()
                        if m == -np.inf:
                            continue
                        p = np.exp(y - m)
                        out[t, head], lse[t, head] = (p / p.sum()) @ v[at], m + np.log(p.sum())
        return out, lse

    def weigh(self, lse, decay, weight=None):
        """The account after the call, [seqs, kv_heads, max len]; NaN behind the lengths."""
        S = len(self.lens)
        w = np.full((S, self.kv_heads, max(self.lens, default=0)), np.nan)
        for s in range(S):
            n = self.lens[s]
            for h in range(self.kv_heads):
                got = np.zeros(n)
                for head in range(h * self.group, (h + 1) * self.group):
                    x, see = self.scores(s, head)
                    z = lse[self.offset[s]: self.offset[s + 1], head][:, None]
                    p = np.where(see & (z > -np.inf), np.exp(np.where(see & (z > -np.inf), x - z, -np.inf)), 0)
                    got += p.sum(0)
                w[s, h, :n] = got + (0 if weight is None else decay * weight[s, h, :n].double().numpy())
        return w


def evict_order(weight, pos, length, protect, recent_from):
    """Slots in the order in which they are kept."""
    def key(j):
        w = float(weight[j])
        cls = 0 if j < protect else 1 if pos[j] >= recent_from else 2
        return (cls, 0.0 if cls == 0 else math.inf if math.isnan(w) else -w if not math.isinf(w) else (-1e300 if w > 0 else 1e300), j)
    return sorted(range(length), key=key)


def evict(weight, pos, length, budget, protect, recent_from):
    """(new length, slot that each slot of the front is filled from) of one head of a sequence."""
    protect = min(length, max(0, protect))
    new = min(length, max(protect, max(0, budget)))
    kept = sorted(evict_order(weight, pos, length, protect, recent_from)[:new])
    src = list(range(new))
    gaps = [j for j in range(new) if j not in set(kept)]
    for gap, j in zip(gaps, [j for j in kept if j >= new]):
        src[gap] = j
    return new, src
