"""Performance cases of the rows of a paged KV cache: written with norm and rotation, held in 4 bits, read back, attended to.

A user holds the blocks of a pool, a block table and the sequences' lengths.  The pool is either K and V in 16 bits
(``PagedCache``) or one tensor of bytes with K and V in 4 bits (``PackedCache``).  One pass is:

  write   new tokens' queries and keys get the norm of their heads and the rotation by position, and keys and values
          go into the slots of a 16-bit cache; returns the queries and the pool
  pack    the same into a 4-bit cache, and the new rows read back from it; returns queries, keys and values
  read    sequences of a 4-bit cache as 16-bit rows, as where they go back into a 16-bit one
  attend  attention over a 4-bit cache: single tokens, trees of drafted tokens, chunks of prompts

The 4 bits are those of the microscaling formats: sign, two bits of exponent, one of mantissa (0, 0.5, 1, 1.5, 2, 3, 4, 6),
and a power of two for each 32 elements of a head, in a byte of its own: 2^e with the least e for which the largest of the
32 is at most 7 * 2^e.  A (block, head) is its keys' bytes, its values' bytes, its keys' scales, its values' scales, each
[slots, ...]; the lower four bits of a byte are the earlier element.

Lengths, rows, documents and trees follow from the case, values and the order of the blocks from the seed.  Slots past a
sequence's length hold bytes of ones, as a reused block may.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
NEVER = 1 << 30  # a row_start behind every slot: a padding row, which sees nothing of its own
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ cases
def _rows_case(name, kind, seqs, rows_lo, rows_hi, past, q_heads, kv_heads, dim, dtype, page=16, norm=True, rot=1.0, base=10000.0,
               axes=0, interleaved=False, far=0):
    """New rows behind 0 to `past` older slots.  rot: the rotated part of a head; axes: positions of a row (0: one, its slot
    or, with `far`, one up to that); base: of the rotation's frequencies."""
    c = dict(kind=kind, seqs=seqs, rows_lo=rows_lo, rows_hi=rows_hi, past=past, q_heads=q_heads, kv_heads=kv_heads, dim=dim,
             dtype=dtype, page=page, norm=norm, rot=rot, base=base, axes=axes, interleaved=interleaved, far=far)
    return dict(c, name=name) if name else c


def _read(name, seqs, len_lo, len_hi, kv_heads, dim, dtype, page=16):
    c = dict(kind="read", seqs=seqs, len_lo=len_lo, len_hi=len_hi, kv_heads=kv_heads, dim=dim, dtype=dtype, page=page)
    return dict(c, name=name) if name else c


def _attend(name, form, seqs, len_lo, len_hi, rows_lo, rows_hi, q_heads, kv_heads, dim, dtype, page=16, softcap=0.0,
            bias=False, docs=0, prefix=0):
    c = dict(kind="attend", form=form, seqs=seqs, len_lo=len_lo, len_hi=len_hi, rows_lo=rows_lo, rows_hi=rows_hi,
             q_heads=q_heads, kv_heads=kv_heads, dim=dim, dtype=dtype, page=page, softcap=softcap, bias=bias, docs=docs,
             prefix=prefix)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decode step's tokens of a batch: all latency
        _rows_case("write_token", "write", 64, 1, 1, 1023, 32, 8, 128, "bf16"),
        # chunks of unlike prompts, far positions as after evictions
        _rows_case("write_chunk", "write", 24, 1, 1024, 2048, 32, 8, 128, "bf16", base=500000.0, far=1 << 24),
        # frames of a video: positions in time, height and width, pairs side by side, part of the head, no norm
        _rows_case("write_axes", "write", 2, 4000, 4097, 500, 16, 16, 64, "f16", page=32, norm=False, rot=0.75, axes=3, interleaved=True),
        # a decode step's tokens into a cache of 4 bits
        _rows_case("pack_token", "pack", 64, 1, 1, 1023, 32, 8, 128, "bf16"),
        # chunks of unlike prompts into it
        _rows_case("pack_chunk", "pack", 24, 1, 1024, 2048, 32, 8, 128, "bf16", base=500000.0, far=1 << 24),
        # four claims of 80 blocks brought back
        _read("read_probe", 4, 1, 1280, 2, 64, "f16"),
        # long ones of wide heads, blocks of 64 tokens
        _read("read_long", 6, 20000, 65536, 4, 256, "bf16", page=64),
        # one token for each of four pools of 80 blocks: all latency
        _attend("attend_probe", "tree", 4, 1, 1280, 1, 1, 8, 2, 64, "f16"),
        # a scheduler's decode step over unlike lengths
        _attend("attend_batch", "tree", 64, 1, 8192, 1, 1, 32, 8, 128, "bf16"),
        # pools of 16,384 blocks, one sequence each
        _attend("attend_long", "tree", 5, 250001, 262144, 1, 1, 32, 8, 128, "bf16"),
        # drafted trees verified for a batch
        _attend("attend_tree", "tree", 40, 700, 8192, 12, 64, 32, 8, 128, "bf16"),
        # one more chunk of a long prompt, capped scores
        _attend("attend_chunk", "chunk", 1, 32768, 32768, 2048, 2048, 32, 8, 128, "bf16", softcap=50.0),
    ]


def _log(rng, a, b):
    """An integer of [a, b], spread over its logarithm."""
    return min(b, max(a, int(round(a * (b / a) ** rng.random()))))


def draw(rng: random.Random):
    kind = rng.choice(("write", "write", "pack", "pack", "read", "decode", "decode", "tree", "chunk", "docs"))
    kv_heads = rng.choice((1, 2, 4, 8))
    group = rng.choice((1, 2, 3, 4, 5, 8))
    dim = rng.choice((64, 128, 128, 256))
    dtype = rng.choice(("bf16", "f16"))
    page = rng.choice((16, 16, 32, 64))
    if kind in ("write", "pack"):
        seqs = _log(rng, 1, 64)
        hi = _log(rng, 1, max(1, min(8192, (1 << 25) // (seqs * (group + 2) * kv_heads * dim))))
        axes = rng.choice((0, 0, 2, 3))
        return _rows_case(None, kind, seqs, rng.randint(1, hi), hi, rng.randint(0, min(2048, 65536 // seqs)), group * kv_heads, kv_heads,
                          dim, dtype, page, norm=rng.random() < 0.6, rot=rng.choice((0.0, 0.25, 0.5, 1.0, 1.0)),
                          base=rng.choice((1e4, 5e5)), axes=axes, interleaved=rng.random() < 0.4, far=0 if axes else rng.choice((0, 1 << 24)))
    if kind == "read":
        seqs = _log(rng, 1, 64)
        hi = _log(rng, 17, min(262144, (1 << 27) // (seqs * kv_heads * dim)))
        return _read(None, seqs, rng.randint(1, hi), hi, kv_heads, dim, dtype, page)
    cap = rng.choice((0.0, 0.0, 20.0, 50.0))
    bias = rng.random() < 0.3
    if kind == "decode":
        seqs = _log(rng, 1, 64)
        hi = _log(rng, 17, min(262144, (1 << 20) // seqs, (1 << 30) // (seqs * kv_heads * dim)))
        return _attend(None, "tree", seqs, rng.randint(1, hi), hi, 1, 1, group * kv_heads, kv_heads, dim, dtype, page, cap, bias)
    heads = group * kv_heads * dim  # what a pair of a row and a slot costs
    if kind == "tree":
        seqs = _log(rng, 1, 32)
        rows = rng.randint(2, 64)
        hi = _log(rng, 80, 65536 // max(seqs, 4))
        return _attend(None, "tree", seqs, rng.randint(64, hi), hi, rng.randint(1, rows), rows, group * kv_heads, kv_heads,
                       dim, dtype, page, cap, bias)
    if kind == "chunk":
        seqs = _log(rng, 1, 24)
        rows = _log(rng, 5, 4096 // seqs)
        hi = rows + _log(rng, 1, max(1, min(16384 // seqs, (1 << 37) // (heads * seqs * rows) - rows)))
        return _attend(None, "chunk", seqs, rng.randint(rows, hi), hi, rng.randint(1, rows), rows, group * kv_heads, kv_heads,
                       dim, dtype, page, cap, bias)
    seqs = rng.randint(1, 3)
    rows = _log(rng, 100, min(4096, int(((1 << 37) / (heads * seqs)) ** 0.5)))
    return _attend(None, "chunk", seqs, rng.randint(rows // 2, rows), rows, rows, rows, group * kv_heads, kv_heads, min(dim, 128),
                   dtype, page, cap, bias, docs=rng.randint(1, 12), prefix=rng.randint(0, rows // 2))


# ------------------------------------------------------------------------------- what follows from a case
def _shape(case):
    """Lengths, rows and masks of a case's sequences, as lists."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    S = case["seqs"]
    if case["kind"] in ("write", "pack"):
        lo, hi = case["rows_lo"], case["rows_hi"]
        rows = [rng.randint(lo, hi) for _ in range(S)]
        rows[0] = hi
        if S > 1:
            rows[1] = lo
        lens = [r + rng.randint(0, case["past"]) for r in rows]
        return dict(lens=lens, rows=rows, max_len=max(lens), first=[rng.randrange(case["far"]) if case["far"] else n - r for n, r in zip(lens, rows)])
    lo, hi = case["len_lo"], case["len_hi"]
    lens = [rng.randint(lo, hi) for _ in range(S)]
    lens[0] = hi
    if S > 1:
        lens[1] = lo
    if case["kind"] == "read":
        return dict(lens=lens, rows=lens, max_len=hi)
    rows = [min(n, rng.randint(case["rows_lo"], case["rows_hi"])) for n in lens]
    rows[0] = min(lens[0], case["rows_hi"])
    sh = dict(lens=lens, max_len=hi, rows=rows, max_rows=max(rows), parent=None, row_start=None, prefix=None)
    if case["form"] == "tree" and case["rows_hi"] > 1:
        sh["parent"] = [rng.randint(max(-1, i - 8), i - 1) for n in rows for i in range(n)]
    if case["docs"]:
        start, prefix = [], []
        for n, r in zip(lens, rows):
            cuts = sorted({0} | {rng.randrange(n) for _ in range(case["docs"] - 1)})
            at = [max(c for c in cuts if c <= n - r + i) for i in range(r)]
            pad = r // 50  # the chunk's last rows are padding
            start += at[: r - pad] + [NEVER] * pad
            prefix.append(min(case["prefix"], n) if len(prefix) % 2 == 0 else 0)
        sh.update(row_start=start, prefix=prefix)
    return sh


def _visible(sh):
    """Pairs of a row and a slot that it sees, over all sequences."""
    pairs, at = 0, 0
    for s, (n, r) in enumerate(zip(sh["lens"], sh["rows"])):
        seen = []
        for i in range(r):
            if sh["parent"] is not None:
                p = sh["parent"][at + i]
                seen.append(1 + (seen[p] if p >= 0 else 0))
                pairs += n - r + seen[i]
                continue
            last, first = n - r + i, 0 if sh["row_start"] is None else sh["row_start"][at + i]
            pre = 0 if sh["prefix"] is None else sh["prefix"][s]
            pairs += min(pre, n) + max(0, last + 1 - max(first, pre))
        at += r
    return pairs


def _rotated(case):
    """Elements of a head that turn, a multiple of 16."""
    return int(case["dim"] * case["rot"]) // 16 * 16


def work(case):
    sh = _shape(case)
    H, D, T, slots = case["kv_heads"], case["dim"], sum(sh["rows"]), sum(sh["lens"])
    table, held = 4 / case["page"], 2 * H * (D / 2 + D / 32)  # of a slot: its share of the table, its bytes of 4 bits
    if case["kind"] in ("write", "pack"):
        Q = case["q_heads"]
        each = 2 * Q * D * 2 + 2 * H * D * 2 + table + (4 * max(1, case["axes"]) if case["axes"] or case["far"] else 0)
        # a norm is 4 operations an element, a rotation 3; keys and values come back once more from the 4 bits
        f = T * (Q + H) * (4 * D * case["norm"] + 3 * _rotated(case))
        return {"bytes": T * (each + (2 * H * D * 2 if case["kind"] == "write" else 2 * held + 2 * H * D * 2)), "flops": f}
    if case["kind"] == "read":
        return {"bytes": T * (table + held + 2 * H * D * 2), "flops": T * 2 * H * D}
    Q = case["q_heads"]
    return {"bytes": slots * (table + held) + 4 * T * Q * D + 4 * T * Q, "flops": 4 * _visible(sh) * Q * D}


# ------------------------------------------------------------------------------------------------ inputs
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _parts(pool, page, dim):
    """Keys' bytes, values' bytes, keys' scales and values' scales, [blocks, heads, slots, ...]."""
    c, s = page * dim // 2, page * dim // 32
    return tuple(p.unflatten(-1, (page, -1)) for p in pool.split([c, c, s, s], dim=-1))


def _packed_pool(g, blocks, H, page, D, dtype):
    """Keys with channels of unlike size, and values, in 4 bits."""
    pool = torch.empty(blocks, H, page * (D + D // 16), dtype=torch.uint8, device=DEV)
    kc, vc, ks, vs = _parts(pool, page, D)
    channel = torch.empty(H, 1, D, device=DEV).normal_(generator=g).mul_(0.4).exp_()
    step = max(1, (1 << 25) // (H * page * D))
    for b in range(0, blocks, step):
        n = min(step, blocks - b)
        x = torch.empty(2, n, H, page, D, device=DEV).normal_(generator=g)
        x[0] *= channel
        code, scale, _ = _quantised(x, dtype)
        kc[b: b + n], vc[b: b + n], ks[b: b + n], vs[b: b + n] = code[0], code[1], scale[0], scale[1]
    return pool


def prepare(case, seed):
    sh = _shape(case)
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    S, H, D, page, dtype = case["seqs"], case["kv_heads"], case["dim"], case["page"], TYPES[case["dtype"]]
    kind, T = case["kind"], sum(sh["rows"])
    pages = -(-sh["max_len"] // page)
    blocks = S * pages + 3
    table = torch.randperm(blocks, generator=g, device=DEV)[: S * pages].to(torch.int32).reshape(S, pages)
    length = _ints(sh["lens"])
    offset = [0]
    for r in sh["rows"]:
        offset.append(offset[-1] + r)
    st = dict(case=dict(case), table=table, length=length, max_len=sh["max_len"], row_offset=_ints(offset), dtype=dtype, rows=T)
    if kind == "write":
        st["k"] = torch.empty(blocks, page, H, D, dtype=dtype, device=DEV).normal_(generator=g)
        st["v"] = torch.empty(blocks, page, H, D, dtype=dtype, device=DEV).normal_(generator=g)
    elif kind == "pack":
        st["pool"] = torch.randint(0, 256, (blocks, H, page * (D + D // 16)), generator=g, device=DEV, dtype=torch.uint8)
    else:
        st["pool"] = _packed_pool(g, blocks, H, page, D, dtype)
        # what lies behind a sequence's length in its last block is not the sequence's
        last = table.gather(1, ((length - 1) // page).long()[:, None])[:, 0].long()
        behind = torch.arange(page, device=DEV)[None] > ((length - 1) % page)[:, None]
        for part in _parts(st["pool"], page, D):
            part[last] = part[last].masked_fill(behind[:, None, :, None], 255)
    if kind in ("write", "pack"):
        Q, R = case["q_heads"], _rotated(case)
        # the rows of a fused projection: queries, keys and values side by side
        x = torch.empty(T, Q + 2 * H, D, device=DEV).normal_(generator=g)
        x[:, :-H] *= torch.empty(Q + H, D, device=DEV).normal_(generator=g).mul_(0.4).exp_()  # channels of unlike size
        x = x.to(dtype)
        st.update(q=x[:, :Q], new_k=x[:, Q: Q + H], new_v=x[:, Q + H:], q_norm=None, k_norm=None, freq=None, axis=None, position=None)
        if case["norm"]:
            for f in ("q_norm", "k_norm"):
                st[f] = (1 + 0.2 * torch.empty(D, device=DEV).normal_(generator=g)).to(dtype)
        if R:
            half = torch.arange(R // 2, device=DEV, dtype=torch.float64)
            st["freq"] = torch.pow(torch.tensor(case["base"], dtype=torch.float64, device=DEV), -2 * half / R).float()
        seq, i = _rows(st)
        first = torch.tensor(sh["first"], device=DEV)[seq] + i
        if R and case["axes"]:
            # frames of 12 by 20 patches: time goes on, height and width start again
            at = (first // 240, first // 20 % 12, first % 20)[: case["axes"]]
            st.update(position=torch.stack(at).to(torch.int32), axis=(torch.arange(R // 2, device=DEV) % case["axes"]).to(torch.int32))
        elif R and case["far"]:
            st["position"] = first.to(torch.int32)
    if kind == "attend":
        Q = case["q_heads"]
        q = torch.empty(T, Q, D, device=DEV).normal_(generator=g)
        q *= 10.0 if case["softcap"] else 2.0  # scores that reach the cap, or a softmax of ordinary width
        st.update(q=q.to(dtype), max_rows=sh["max_rows"], parent=None, row_start=None, prefix=None, slope=None,
                  scale=1 / math.sqrt(D), softcap=case["softcap"])
        for f in ("parent", "row_start", "prefix"):
            if sh[f] is not None:
                st[f] = _ints(sh[f])
        if case["bias"]:
            st["slope"] = torch.exp2(-8.0 * torch.arange(1, Q + 1, device=DEV) / Q)
    if own:
        import paper_2605_24259_amd as rkc
        if kind == "write":
            st["cache"] = rkc.PagedCache(st["k"], st["v"], table)
        else:
            st["cache"] = rkc.PackedCache(st["pool"], table, page_tokens=page, head_dim=D, dtype=dtype)
    return st


# -------------------------------------------------------------------------------------------- plain forms
def _rows(st):
    """Of each row: its sequence and its place there."""
    t = torch.arange(st["rows"], device=DEV)
    seq = torch.searchsorted(st["row_offset"][1:].long(), t, right=True)
    return seq, t - st["row_offset"].long()[seq]


def _places(st):
    """Of each row: its block, and its slot there."""
    seq, i = _rows(st)
    n = (st["row_offset"][1:] - st["row_offset"][:-1]).long()
    slot = st["length"].long()[seq] - n[seq] + i
    page = st["case"]["page"]
    return st["table"].long()[seq, slot // page], slot % page, slot


def _normed(st, x, weight):
    if weight is None:
        return x
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.to(x.dtype)


def _turned(st, x):
    """The rotation of each pair by its frequency times the row's position; angles in 64 bits."""
    freq = st["freq"]
    if freq is None:
        return x
    at = _places(st)[2][None] if st["position"] is None else st["position"].reshape(-1, st["rows"])
    at = at.double()
    at = at[0][:, None] if st["axis"] is None else at[st["axis"].long()].T
    angle = (at * freq.double())[:, None]
    cos, sin = torch.cos(angle).to(x.dtype), torch.sin(angle).to(x.dtype)
    R = 2 * freq.shape[0]
    y = x[..., :R]
    if st["case"]["interleaved"]:
        a, b = y[..., 0::2], y[..., 1::2]
        y = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    else:
        a, b = y[..., : R // 2], y[..., R // 2:]
        y = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    return torch.cat((y, x[..., R:]), dim=-1)


def _quantised(x, dtype):
    """Bytes of two elements, bytes of scales, and what they stand for, of x in 32 bits: [..., D] -> [..., D / 2], [..., D / 32],
    [..., D].  The last steps of a half go to the even code; past 7 times the largest scale, 6 times it is held."""
    x = x.unflatten(-1, (-1, 32))
    most = x.abs().amax(-1)
    # 2^e with the least e for which most <= 7 * 2^e: a mantissa past 1.75 carries into the exponent
    e = (((most.view(torch.int32) + 0x1FFFFF) >> 23) - 2).clamp(1, 127 + (13 if dtype == torch.float16 else 125))
    y = x * ((254 - e) << 23).to(torch.int32).view(torch.float32)[..., None]
    m = y.abs()
    at = (m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5)
    code = at + (torch.signbit(y).to(torch.uint8) << 3)
    code = code.flatten(-2)
    code = code[..., 0::2] | (code[..., 1::2] << 4)
    e = e.to(torch.uint8)
    return code, e, _values(code, e)


def _values(code, scale):
    """[..., D / 2] and [..., D / 32] bytes -> [..., D] in 32 bits."""
    c = torch.arange(8, device=DEV)
    of = torch.where(c < 2, c * 0.5, torch.exp2((c // 2 - 1).float()) * (1 + 0.5 * (c % 2)))
    of = torch.cat((of, -of))
    b = torch.arange(256, device=DEV)
    pair = torch.stack((of[b % 16], of[b // 16]), dim=-1)
    x = pair[code.long()].flatten(-2).unflatten(-1, (-1, 32))
    by = (scale.to(torch.int32) << 23).view(torch.float32)
    return (x * by[..., None]).flatten(-2)


def _plain_write(st):
    block, slot, _ = _places(st)
    q = _turned(st, _normed(st, st["q"].float(), st["q_norm"])).to(st["dtype"])
    k = _turned(st, _normed(st, st["new_k"].float(), st["k_norm"])).to(st["dtype"])
    st["k"][block, slot], st["v"][block, slot] = k, st["new_v"]
    return {"q": q, "k": st["k"], "v": st["v"]}


def _plain_pack(st):
    block, slot, _ = _places(st)
    q = _turned(st, _normed(st, st["q"].float(), st["q_norm"])).to(st["dtype"])
    # in 64 bits up to the rounding, as values next to a border between two codes would else go either way
    k = _turned(st, _normed(st, st["new_k"].double(), st["k_norm"])).float()
    parts = _parts(st["pool"], st["case"]["page"], st["case"]["dim"])
    (kc, ks, _), (vc, vs, _) = _quantised(k, st["dtype"]), _quantised(st["new_v"].float(), st["dtype"])
    for part, x in zip(parts, (kc, vc, ks, vs)):
        part.transpose(1, 2)[block, slot] = x
    k, v = _plain_read(st)
    return {"q": q, "k": k, "v": v}


def _plain_read(st):
    block, slot, _ = _places(st)
    kc, vc, ks, vs = (part.transpose(1, 2)[block, slot] for part in _parts(st["pool"], st["case"]["page"], st["case"]["dim"]))
    return _values(kc, ks).to(st["dtype"]), _values(vc, vs).to(st["dtype"])


def _padded(st, x, fill):
    """[T, ...] -> [S, max_rows, ...]"""
    seq, i = _rows(st)
    y = x.new_full((st["length"].shape[0], st["max_rows"]) + tuple(x.shape[1:]), fill)
    y[seq, i] = x
    return y


def _gathered(st, which):
    """The sequences' keys (0) or values (1) in order, [S, H, max_len, D] in 32 bits; nothing behind their lengths."""
    n = st["max_len"]
    parts = _parts(st["pool"], st["case"]["page"], st["case"]["dim"])
    code, scale = (parts[i][st["table"].long()].transpose(2, 3).flatten(1, 2)[:, :n] for i in (which, 2 + which))
    held = torch.arange(n, device=DEV)[None] < st["length"][:, None]
    x = torch.where(held[:, :, None, None], _values(code, scale), torch.zeros((), device=DEV))
    return x.transpose(1, 2).contiguous()


def _seen(st):
    """Which slots each row sees and how far they are, [S, max_rows, max_len]."""
    n, R = st["max_len"], st["max_rows"]
    length, rows = st["length"].long(), (st["row_offset"][1:] - st["row_offset"][:-1]).long()
    base = (length - rows)[:, None, None]
    slot = torch.arange(n, device=DEV)[None, None]
    i = torch.arange(R, device=DEV)[None, :, None]
    start = 0 if st["row_start"] is None else _padded(st, st["row_start"].long(), 0)[:, :, None]
    prefix = 0 if st["prefix"] is None else st["prefix"].long()[:, None, None]
    at, where = base + i, slot
    if st["parent"] is None:
        see = ((slot >= start) & (slot <= at)) | (slot < prefix)
    else:
        p = _padded(st, st["parent"].long(), -1)
        a = torch.eye(R, device=DEV) + (p[:, :, None] == torch.arange(R, device=DEV)[None, None]).float()
        a = (a @ a).clamp(max=1)
        a = (a @ a).clamp(max=1)
        a = (a @ a).clamp(max=1)
        a = (a @ a).clamp(max=1)
        a = (a @ a).clamp(max=1)
        a = (a @ a).clamp(max=1)  # chains of up to 64
        depth = a.sum(-1).long() - 1
        drafted = slot - base
        inside = (drafted >= 0) & (drafted < R)
        j = drafted.clamp(0, R - 1)
        see = torch.where(inside, a.gather(2, j.expand(-1, R, -1)) > 0, ((slot >= start) | (slot < prefix)) & (drafted < 0))
        at = base + depth[:, :, None]
        where = torch.where(inside, base + depth[:, None, :].gather(2, j), slot)
    return see & (slot < length[:, None, None]) & (i < rows[:, None, None]), (at - where).abs()


def _scores(st):
    """Scores of each row and head against each slot, -inf where unseen: [S, H, max_rows * group, max_len]."""
    S, R, n, H, D = st["length"].shape[0], st["max_rows"], st["max_len"], st["case"]["kv_heads"], st["case"]["dim"]
    G = st["q"].shape[1] // H
    q = _padded(st, st["q"].float(), 0.0).reshape(S, R, H, G, D).permute(0, 2, 1, 3, 4).reshape(S, H, R * G, D)
    s = q.contiguous() @ _gathered(st, 0).transpose(2, 3).contiguous()
    s *= st["scale"]
    if st["softcap"]:
        s = torch.tanh(s / st["softcap"]) * st["softcap"]
    see, far = _seen(st)
    s = s.view(S, H, R, G, n)
    if st["slope"] is not None:
        s = s - st["slope"].view(1, H, 1, G, 1) * far[:, None, :, None].float()
    return s.masked_fill(~see[:, None, :, None], float("-inf")).view(S, H, R * G, n)


def _back(st, x):
    """[S, H, max_rows * group, ...] -> [T, H * group, ...]"""
    seq, i = _rows(st)
    H, R = x.shape[1], st["max_rows"]
    x = x.reshape((x.shape[0], H, R, x.shape[2] // R) + tuple(x.shape[3:]))
    x = x[seq, :, i]
    return x.flatten(1, 2)


def _plain_attend(st):
    s = _scores(st)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), torch.zeros((), device=DEV), top)
    s = torch.exp(s - top)
    total = s.sum(-1, keepdim=True)
    o = s @ _gathered(st, 1)
    o = torch.where(total == 0, torch.zeros((), device=DEV), o / total)
    lse = (top + torch.log(total))[..., 0]
    return {"out": _back(st, o).to(st["q"].dtype), "lse": _back(st, lse)}


def run(st):
    kind = st["case"]["kind"]
    if not own:
        if kind == "read":
            k, v = _plain_read(st)
            return {"k": k, "v": v}
        return {"write": _plain_write, "pack": _plain_pack, "attend": _plain_attend}[kind](st)
    cache, at = st["cache"], (st["row_offset"], st["length"])
    if kind == "attend":
        out, lse = cache.attend(st["q"], *at, max_rows=st["max_rows"], max_len=st["max_len"], scale=st["scale"], softcap=st["softcap"],
                                slope=st["slope"], prefix=st["prefix"], row_start=st["row_start"], parent=st["parent"])
        return {"out": out, "lse": lse}
    if kind == "read":
        k, v = cache.read(*at, rows=st["rows"])
        return {"k": k, "v": v}
    q = cache.store(st["new_k"], st["new_v"], *at, q=st["q"], q_norm=st["q_norm"], k_norm=st["k_norm"], eps=EPS, freq=st["freq"],
                    position=st["position"], axis=st["axis"], interleaved=st["case"]["interleaved"])
    if kind == "write":
        return {"q": q, "k": st["k"], "v": st["v"]}
    k, v = cache.read(*at, rows=st["rows"])
    return {"q": q, "k": k, "v": v}


# ------------------------------------------------------------------------------------ the same in 64 bits
def _exact_rows(case, st, sh, x, weight):
    """Norm and rotation of [T, heads, D], pair by pair of the definition."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS) * weight.double()
    if st["freq"] is None:
        return x
    pairs = st["freq"].shape[0]
    if st["position"] is None:
        p = torch.cat([torch.arange(n - r, n, device=DEV) for n, r in zip(sh["lens"], sh["rows"])])[None]
    else:
        p = st["position"].reshape(-1, x.shape[0])
    y = x.clone()
    for j in range(pairs):
        a, b = (2 * j, 2 * j + 1) if case["interleaved"] else (j, j + pairs)
        t = p[0 if st["axis"] is None else j % case["axes"]].double() * st["freq"][j].double()
        z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.ones_like(t), t)[:, None]
        y[..., a], y[..., b] = z.real, z.imag
    return y


def _exact_held(x, dtype):
    """What 4 bits hold of x: the nearest of the sixteen times 2^e, of two as near the one with the even code."""
    x = x.float().double().unflatten(-1, (-1, 32))
    m, e = torch.frexp(x.abs().amax(-1))
    e = torch.where(m <= 7 / 8, e - 3, e - 2).clamp(-126, 13 if dtype == torch.float16 else 125)
    by = torch.exp2(e.double())[..., None]
    best, value = torch.full_like(x, 1e300), torch.zeros_like(x)
    for code in (0, 2, 4, 6, 1, 3, 5, 7):  # even codes first: another has to be nearer
        v = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)[code]
        off = (x.abs() / by - v).abs()
        value = torch.where(off < best, torch.full_like(x, v), value)
        best = torch.minimum(best, off)
    return (torch.copysign(value, x) * by).flatten(-2)


def _exact_slots(case, st, s, h, n):
    """Keys and values of a sequence's first n slots of head h."""
    page, D = case["page"], case["dim"]
    own_blocks = st["pool"][st["table"][s, : -(-n // page)].long(), h]
    got = []
    for at, scales in ((0, page * D), (page * D // 2, page * D + page * D // 32)):
        b = own_blocks[:, at: at + page * D // 2].reshape(-1, D // 2)[:n]
        c = torch.stack((b & 15, b >> 4), dim=-1).reshape(n, D).long()
        e, m = (c & 7) >> 1, (c & 1).double()
        x = torch.where(e == 0, m / 2, (1 + m / 2) * torch.exp2((e - 1).double())) * (1 - 2 * (c >> 3)).double()
        by = own_blocks[:, scales: scales + page * D // 32].reshape(-1, D // 32)[:n].double() - 127
        got.append(x * torch.exp2(by).repeat_interleave(32, dim=1))
    return got


def exact(case, seed):
    sh, st = _shape(case), prepare(case, seed)
    H, D, page, n_rows = case["kv_heads"], case["dim"], case["page"], st["rows"]
    if case["kind"] in ("write", "pack"):
        q = _exact_rows(case, st, sh, st["q"], st["q_norm"])
        k, v = _exact_rows(case, st, sh, st["new_k"], st["k_norm"]), st["new_v"].double()
        if case["kind"] == "pack":
            return {"q": q, "k": _exact_held(k, st["dtype"]), "v": _exact_held(v, st["dtype"])}
        pk, pv, at = st["k"].double(), st["v"].double(), 0
        for s, (n, r) in enumerate(zip(sh["lens"], sh["rows"])):
            slot = torch.arange(n - r, n, device=DEV)
            block = st["table"][s].long()[slot // page]
            pk[block, slot % page], pv[block, slot % page] = k[at: at + r], v[at: at + r]
            at += r
        return {"q": q, "k": pk, "v": pv}
    if case["kind"] == "read":
        k = torch.zeros(n_rows, H, D, dtype=torch.float64, device=DEV)
        v, at = torch.zeros_like(k), 0
        for s, n in enumerate(sh["lens"]):
            for h in range(H):
                k[at: at + n, h], v[at: at + n, h] = _exact_slots(case, st, s, h, n)
            at += n
        return {"k": k, "v": v}
    G = case["q_heads"] // H
    out = torch.zeros(n_rows, case["q_heads"], D, dtype=torch.float64, device=DEV)
    lse = torch.full((n_rows, case["q_heads"]), float("-inf"), dtype=torch.float64, device=DEV)
    at = 0
    for s, (n, r) in enumerate(zip(sh["lens"], sh["rows"])):
        base, slot = n - r, torch.arange(n, device=DEV)
        see = torch.zeros(r, n, dtype=torch.bool, device=DEV)
        place, mine = slot.clone(), base + torch.arange(r, device=DEV)
        if sh["parent"] is not None:
            line = []
            for i in range(r):
                p = sh["parent"][at + i]
                line.append((line[p] if p >= 0 else []) + [i])
            drafts = torch.zeros(r, r, dtype=torch.bool)
            for i, path in enumerate(line):
                drafts[i, path] = True
            see[:, :base] = True
            see[:, base:] = drafts.to(DEV)
            mine = base + torch.tensor([len(p) - 1 for p in line], device=DEV)
            place[base:] = mine
        else:
            first = torch.zeros(r, dtype=torch.long, device=DEV) if st["row_start"] is None else st["row_start"][at: at + r].long()
            see = (slot[None] >= first[:, None]) & (slot[None] <= mine[:, None])
            if sh["prefix"] is not None:
                see[:, : sh["prefix"][s]] = True
        far = (mine[:, None] - place[None]).abs().double()
        for h in range(H):
            kk, vv = _exact_slots(case, st, s, h, n)
            for j in range(h * G, (h + 1) * G):
                x = (st["q"][at: at + r, j].double() @ kk.T) * st["scale"]
                if st["softcap"]:
                    x = st["softcap"] * torch.tanh(x / st["softcap"])
                if st["slope"] is not None:
                    x = x - st["slope"][j].double() * far
                x = x.masked_fill(~see, float("-inf"))
                z = torch.logsumexp(x, -1)
                p = torch.where(z[:, None] > float("-inf"), torch.exp(x - z[:, None]), torch.zeros_like(x))
                out[at: at + r, j], lse[at: at + r, j] = p @ vv, z
        at += r
    return {"out": out, "lse": lse}
