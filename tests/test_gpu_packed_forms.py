"""Attention over a cache of 4 bits in the forms that only large batches take: many sequences over the blocks of one pool, which
keeps the plain implementation small.  Tolerances as in test_gpu_cache.py."""
import numpy as np
import pytest
import torch

from tests import packed_reference as ref
from tests.gpu_util import say
from tests.test_gpu_cache import check_attend, ints, mask
from tests.test_gpu_packed import packed_cache
from tests.test_packed_plan import lib, plan_of  # noqa: F401

pytestmark = pytest.mark.gpu


def shared(seed, lens, rows, *, kv_heads, group, dim, dtype="bfloat16", page=16, marks=(), softcap=0.0, bias=False, parent=None, row_start=None,
           prefix=None):
    """Sequences whose tables name the same blocks, each in an order of its own; `marks`: block, slot and head of what is no number."""
    c = ref.Packed(seed, [-(-max(lens) // page) * page], [1], kv_heads=kv_heads, group=group, dim=dim, dtype=dtype, page=page, softcap=softcap, bias=bias)
    g, rng, mine = torch.Generator().manual_seed(seed), np.random.default_rng(seed), c.table[0, :-1].numpy()
    c.table = torch.from_numpy(np.stack([rng.permutation(mine) for _ in lens]).astype(np.int32))
    c.lens, c.rows, c.offset = list(lens), list(rows), np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    c.q = (torch.randn(sum(rows), kv_heads * group, dim, generator=g) * (8 if softcap else 2)).to(c.dtype)
    c.parent, c.row_start, c.prefix = parent, row_start, prefix
    parts = ref.split(c.pool.numpy(), page, dim)
    for b, i, h in marks:
        parts[2][mine[b], h, i, 0] = 255
    c.pool, c.marks = torch.from_numpy(ref.joined(*parts)), [(int(mine[b]), i, h) for b, i, h in marks]
    return c


def wants(c):
    """(out, lse) of the plain implementation, the heads of a key/value head at once; rows that see a mark get NaN for its head."""
    T, Q = c.q.shape[:2]
    out, lse, q, k, v = np.zeros((T, Q, c.dim)), np.full((T, Q), -np.inf), c.q.double().numpy(), c.k.numpy(), c.v.numpy()
    for s, n in enumerate(c.lens):
        rows, j = slice(int(c.offset[s]), int(c.offset[s + 1])), np.arange(n)
        if not c.rows[s]:
            continue
        see, far = c.seen(s)
        block, at = c.table[s].numpy()[j // c.page], j % c.page
        for h in range(c.kv_heads):
            heads = slice(h * c.group, (h + 1) * c.group)
            x = q[rows, heads] @ k[block, at, h].T * c.scale  # [rows, group, slots]
            if c.softcap:
                x = c.softcap * np.tanh(x / c.softcap)
            if c.slope is not None:
                x -= c.slope[heads].double().numpy()[:, None] * far[:, None]
            x = np.where(see[:, None], x, -np.inf)
            m = x.max(-1, keepdims=True)
            p = np.exp(x - np.where(m == -np.inf, 0, m))
            total = p.sum(-1, keepdims=True)
            with np.errstate(divide="ignore"):
                lse[rows, heads] = (m + np.log(total))[..., 0]
            out[rows, heads] = p @ v[block, at, h] / np.where(total == 0, 1, total)
        for b, i, h in c.marks:
            y = int(np.nonzero(c.table[s].numpy() == b)[0][0]) * c.page + i
            if y < n:
                hit = np.flatnonzero(see[:, y]) + rows.start
                out[hit, h * c.group: (h + 1) * c.group] = lse[hit, h * c.group: (h + 1) * c.group] = np.nan
    return out, lse


def run(c, max_len=None, **kw):
    g = packed_cache(c)
    r = g.attend(c.q.cuda(), ints(c.offset), ints(c.lens), max_len=max_len or max(c.lens), **mask(c, **kw))
    assert not g.status.any().item()
    return r


def lengths(seqs, longest, seed):
    """Of all sizes, the longest and the shortest twice, and an empty sequence."""
    rng = np.random.default_rng(seed)
    n = [int(x) for x in rng.integers(1, longest, seqs)]
    n[:5] = [longest, 1, 0, 1, longest]
    return n


@pytest.mark.parametrize("dtype,dim,seqs,heads,longest", [
    ("bfloat16", 128, 64, 8, 2600), ("float16", 128, 48, 8, 1999), ("bfloat16", 128, 60, 8, 4100), ("bfloat16", 64, 64, 8, 3001),
    ("bfloat16", 128, 70, 8, 1700), ("float16", 64, 170, 8, 1601), ("bfloat16", 128, 33, 8, 2600), ("float16", 128, 65, 8, 4200)])
def test_batches_of_single_tokens(lib, dtype, dim, seqs, heads, longest):  # noqa: F811
    """Whole sequences of more than 1,536 slots, in the order of their lengths and (past 64 of them) not; the last two in parts."""
    say("case batch", dtype, dim, seqs, heads, longest)
    p = plan_of(lib, seqs, heads, dim, 2, 1, longest)
    assert (p.waves == 8 and p.splits == 1) == ((seqs, longest) not in ((33, 2600), (65, 4200))) and p.sorted == (p.splits == 1 and seqs <= 64)
    lens = lengths(seqs, longest, seqs)
    c = shared(seqs, lens, [min(1, n) for n in lens], kv_heads=heads, group=2, dim=dim, dtype=dtype, softcap=20.0 if dim == 64 else 0.0, bias=seqs == 60)
    want = wants(c)
    out, lse = run(c)
    check_attend(c, out, lse, want=want)
    again = run(c)
    assert out.equal(again[0]) and lse.equal(again[1])


NEVER = 1 << 30
WIDE = [  # dim, dtype, sequences, group, rows, longest, what else; 8 key/value heads
    (128, "bfloat16", 32, 4, 50, 700, {}), (128, "float16", 32, 4, 50, 700, dict(softcap=20.0)), (128, "bfloat16", 32, 4, 50, 513, dict(softcap=300.0, bias=True)),
    (128, "float16", 16, 4, 100, 700, dict(bias=True)), (128, "bfloat16", 16, 3, 171, 513, dict(softcap=30.0)), (128, "bfloat16", 32, 4, 50, 700, "tree"),
    (128, "float16", 32, 3, 64, 600, "tree"), (128, "bfloat16", 16, 4, 100, 700, "documents"), (128, "float16", 16, 4, 100, 700, "documents, cap"),
    (256, "bfloat16", 32, 4, 50, 700, {}), (256, "float16", 32, 4, 50, 513, dict(softcap=20.0)), (256, "bfloat16", 32, 5, 40, 600, dict(softcap=300.0, bias=True)),
    (256, "float16", 16, 4, 100, 700, dict(bias=True)), (256, "bfloat16", 32, 4, 50, 700, "tree"), (256, "float16", 16, 4, 100, 700, "documents"),
    (256, "bfloat16", 16, 4, 100, 700, "documents, cap")]


def wide_case(case, marks=()):
    dim, dtype, seqs, group, rows, longest, what = case
    lens, rng = lengths(seqs, longest, seqs + dim), np.random.default_rng(rows)
    ns = [min(n, int(x)) for n, x in zip(lens, rng.integers(1, rows + 1, seqs))]
    ns[0], ns[4] = rows, rows - 1
    kw = dict(what) if isinstance(what, dict) else {}
    if what == "tree":
        from tests.test_gpu_cache import bush
        kw = dict(parent=sum((bush(n, dim + i) for i, n in enumerate(ns)), []), bias=True)
    elif isinstance(what, str):
        # documents of 33 slots, padding rows between; of the first sequence all rows past 60, a tile of its own, see nothing of their own
        start = [NEVER if i % 9 == 0 or (s == 0 and i > 60) else (n - r + i) // 33 * 33 for s, (n, r) in enumerate(zip(lens, ns)) for i in range(r)]
        kw = dict(row_start=start, prefix=[40 * (s % 3 == 1) for s in range(seqs)], softcap=15.0 if "cap" in what else 0.0)
    return shared(dim + rows, lens, ns, kv_heads=8, group=group, dim=dim, dtype=dtype, page=32, marks=marks, **kw)


def check_plan(lib, c):  # noqa: F811
    p = plan_of(lib, len(c.lens), c.kv_heads, c.dim, c.group, max(c.rows), max(c.lens), tree=c.parent is not None)
    assert not p.few and p.rows == 256 and p.splits == 1, (p.few, p.rows, p.splits)


@pytest.mark.parametrize("case", WIDE)
def test_whole_sequences_by_256_rows(lib, case):  # noqa: F811
    """Workgroups of 256 rows that write outputs themselves: one tile of rows and two, the last in part, rows and tiles that see
    nothing; three calls give the same bits."""
    say("case wide", *case)
    c = wide_case(case)
    check_plan(lib, c)
    out, lse = run(c)
    want = wants(c)
    check_attend(c, out, lse, want=want)
    if c.row_start is not None:
        nothing = torch.from_numpy(np.isneginf(want[1]).all(1)).cuda()
        assert nothing.sum() > 40 and out[nothing].eq(0).all()
    for _ in range(2):
        again = run(c)
        assert out.equal(again[0]) and lse.equal(again[1])


@pytest.mark.parametrize("case", [WIDE[i] for i in (0, 1, 2, 5, 7, 8, 9, 10, 11, 13, 15)])
def test_marked_slots_and_256_rows(lib, case):  # noqa: F811
    """Each sequence has the marks at other places: before all rows, between them, behind its length, out of sight of some."""
    say("case wide marks", *case)
    c = wide_case(case, marks=[(1, 5, 0), (9, 31, 3), (15, 16, 3), (4, 0, 7)])
    check_plan(lib, c)
    out, lse = run(c)
    want = wants(c)
    got = np.isnan(want[1])
    assert got.any() and not got.all(1).any() and np.isfinite(want[1]).any()
    check_attend(c, out, lse, want=want)


@pytest.mark.parametrize("softcap,dim,group,rows,dtype", [(20.0, 64, 2, 60, "float16"), (300.0, 128, 2, 60, "bfloat16"), (20.0, 128, 1, 3, "bfloat16"),
                                                          (300.0, 64, 1, 20, "float16"), (20.0, 256, 2, 70, "bfloat16")])
def test_marked_slots_and_caps(softcap, dim, group, rows, dtype):
    """A capped score that is no number stays none, in the other forms too."""
    say("case cap marks", softcap, dim, group, rows, dtype)
    lens = [200, 90, 64]
    c = shared(dim, lens, [min(n, rows) for n in lens], kv_heads=2, group=group, dim=dim, dtype=dtype, softcap=softcap,
               row_start=[50 if i % 2 else 0 for n in lens for i in range(min(n, rows))], marks=[(2, 3, 0), (7, 15, 1)])
    out, lse = run(c)
    want = wants(c)
    assert np.isnan(want[1]).any() and np.isfinite(want[1]).any()
    check_attend(c, out, lse, want=want)


def test_256_rows_captured_and_on_other_streams(lib):  # noqa: F811
    """Replays give the eager bits among other work, three graphs beside each other; two streams at once."""
    say("case wide graph")
    runs = []
    for i in (0, 1, 9, None):
        if i is not None:
            c, max_len = wide_case(WIDE[i]), None
            check_plan(lib, c)
        else:  # in parts, as far as the table goes
            c, max_len = shared(7, [700, 513, 64, 1, 0, 333, 700, 32], [50, 50, 40, 1, 0, 33, 7, 32], kv_heads=8, group=4, dim=128, page=32, softcap=20.0), 8192
            c.table = torch.cat([c.table] * 12, 1).contiguous()
            p = plan_of(lib, 8, 8, 128, 4, 50, max_len)
            assert not p.few and p.rows == 256 and p.splits > 1
        g, q, off, lens = packed_cache(c), c.q.cuda(), ints(c.offset), ints(c.lens)
        m = mask(c, max_len=max_len or max(c.lens))
        want = g.attend(q, off, lens, **m)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = g.attend(q, off, lens, **m)
        runs.append((graph, out, want, g, (q, off, lens), m))
    for turn in range(6):
        for r in runs:
            for x in r[1]:
                x.zero_()
        for r in runs:
            r[0].replay()
        _, _, want, g, at, m = runs[turn % len(runs)]
        eager = g.attend(*at, **m)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, want)), turn
        for _, out, want, *_ in runs:
            assert all(torch.equal(a, b) for a, b in zip(out, want)), turn
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(3):
        got = [r[3].attend(*r[4], stream=streams[i % 2], **r[5]) for i, r in enumerate(runs)]
        torch.cuda.synchronize()
        for (a, b), r in zip(got, runs):
            assert torch.equal(a, r[2][0]) and torch.equal(b, r[2][1]), turn


@pytest.mark.parametrize("dtype,top", [("bfloat16", 252), ("float16", 140)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_every_code_and_scale(dtype, top, dim):
    """Read as the nearest value of the 16-bit type, of two as near the even one: the value itself but for float16 below 2^-24.
    (Half of 2^-24, an odd multiple of it and the like are no float16 numbers.)"""
    import paper_2605_24259_amd as rkc
    say("case codes", dtype, dim)
    f, page = getattr(torch, dtype), 256
    code = (np.arange(dim)[None, None, None] * 7 + np.arange(page)[None, None, :, None]) % 16
    scale = np.minimum(np.arange(page), top - 1)[None, None, :, None] + 1 + np.zeros((1, 1, 1, dim // 32), int)
    parts = [x.astype(np.uint8) for x in (code, (code + 5) % 16, scale, scale[:, :, ::-1])]
    pool = torch.from_numpy(ref.joined(*parts)).cuda()
    c = rkc.PackedCache(pool, ints([[0]]), page_tokens=page, head_dim=dim, dtype=f)
    at = ints([0, page]), ints([page])
    inexact = 0
    for got, codes, scales in zip(c.read(*at, rows=page), (parts[0], parts[1]), (parts[2], parts[3])):
        value = torch.from_numpy(ref.values(codes[0, 0], scales[0, 0]))
        want = value.to(f)  # of 64 bits, rounded once
        assert bits_of(got[:, 0].cpu()).equal(bits_of(want))
        inexact += int((want.double() != value).sum())
        assert dtype == "float16" or torch.equal(want.double(), value)
        assert (want.double() - value).abs().max() <= 2.0 ** -25
    assert (inexact > 0) == (dtype == "float16")
    # and attention over them, a query that sees them all: scores of the values themselves are off by 2^-25 sum |q| at most
    g = torch.Generator().manual_seed(dim)
    q = (torch.randn(1, 2, dim, generator=g) * 1e-4).to(f)
    k, v = (torch.from_numpy(ref.values(a[0, 0], b[0, 0])) for a, b in ((parts[0], parts[2]), (parts[1], parts[3])))
    k[150:], v[:100] = 0, 0
    parts[2][:, :, 150:], parts[0][:, :, 150:], parts[1][:, :, :100] = 1, 0, 0  # the ordinary and the smallest
    c.pool.copy_(torch.from_numpy(ref.joined(*parts)))
    out, lse = c.attend(q.cuda(), ints([0, 1]), ints([page]), max_rows=1)
    s = q[0].double() @ k.T / dim ** 0.5
    p = torch.softmax(s, 1)
    assert (lse[0].double().cpu() - torch.logsumexp(s, 1)).abs().max() <= 2.0 ** -20 * (8 + float(s.abs().max())) + 2.0 ** -25 * float(q.double().abs().sum(-1).max())
    want, half = p @ v, 2.0 ** -8 if dtype == "bfloat16" else 2.0 ** -11
    assert (out[0].double().cpu() - want).abs().max() <= half * float(want.abs().max()) + 2.0 ** -20 * (8 + float(s.abs().max())) * float((p @ v.abs()).max()) + 2.0 ** -24


def bits_of(x):
    return x.contiguous().view(torch.int16)
