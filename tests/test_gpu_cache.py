"""The operators on a paged KV cache against a plain 64-bit implementation, at the sizes and masks where they can go
wrong.

Tolerances.  Scores are sums of 32-bit products: relative to A = |scale| sum |q| |k| (+ cap + slope * distance) their error
is a few units of 2^-24, more with the exponent's base changed and the softmax sum behind it; 2^-20 (8 + A) is allowed
for a logarithm and, relative, for a weight.  Outputs add two roundings to the cache's type (unit roundoff u: 2^-8 or
2^-11), of the weights and of the result: u (sum p |v| + |out|), and what a float16 weight below its normal range loses.
"""
import numpy as np
import pytest

from tests import cache_reference as ref
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

UNIT = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


def gpu_cache(c, dev="cuda"):
    import torch

    import paper_2605_24259_amd as rkc

    def put(x):  # with the strides it has
        y = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=dev)
        return y.copy_(x)
    return rkc.PagedCache(put(c.k), put(c.v), c.table.to(dev))


def ints(x, dev="cuda"):
    import torch
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device=dev)


def mask(c, **kw):
    d = dict(max_rows=max(c.rows, default=0), scale=c.scale, softcap=c.softcap, parent=ints(c.parent),
             slope=None if c.slope is None else c.slope.cuda(), prefix=ints(c.prefix), row_start=ints(c.row_start))
    d.update(kw)
    return d


def reach(c):
    """A of the module's comment, over all scores."""
    far = max(c.lens, default=0) if c.slope is not None else 0
    k = np.nan_to_num(c.k.double().numpy(), nan=0, posinf=0, neginf=0)
    q = np.nan_to_num(c.q.double().numpy(), nan=0, posinf=0, neginf=0)
    if not q.size:
        return 1.0
    return abs(c.scale) * np.linalg.norm(q, axis=-1).max() * np.linalg.norm(k, axis=-1).max() + c.softcap + \
        (0 if c.slope is None else float(c.slope.max()) * far)


def check_attend(c, out, lse, want=None):
    o, z = want or c.attend()
    got, gz = out.double().cpu().numpy(), lse.double().cpu().numpy()
    u, name = UNIT[str(c.dtype).split(".")[1]], str(c.dtype)
    a = 2.0 ** -20 * (8 + reach(c))
    assert np.array_equal(np.isneginf(z), np.isneginf(gz)) and np.array_equal(np.isnan(z), np.isnan(gz))
    ok = np.isfinite(z)
    assert np.all(np.abs(gz - z)[ok] <= a), np.abs(gz - z)[ok].max()
    vmax = np.nan_to_num(np.abs(c.v.double().numpy()), nan=0, posinf=0, neginf=0).max()
    # sum p |v| is at most |v|'s largest element; per element of the output it is bounded by that
    tol = u * (vmax + np.abs(o)) + a * vmax + (2.0 ** -24 * max(c.lens) * vmax if "float16" in name and "b" not in name else 0)
    fin = np.isfinite(o)
    assert np.array_equal(fin, np.isfinite(got)), "other values are not finite"
    assert np.array_equal(np.isnan(o), np.isnan(got)) and np.array_equal(o[~fin & ~np.isnan(o)], got[~fin & ~np.isnan(o)])
    assert np.all(np.abs(got - o)[fin] <= tol[fin]), np.nanmax((np.abs(got - o) / tol)[fin])
    # and as a whole: independent roundings of relative size u, of the weights and of the result
    if fin.any() and np.linalg.norm(o[fin]):
        assert np.linalg.norm((got - o)[fin]) <= (1.5 * u + a) * np.linalg.norm(o[fin]) + 1e-30


def run_attend(c, **kw):
    g = gpu_cache(c)
    r = g.attend(c.q.cuda(), ints(c.offset), ints(c.lens), **mask(c, **kw))
    assert not g.status.any().item()
    return r


def chain(n):
    return list(range(-1, n - 1))


def bush(n, seed=0):
    rng = np.random.default_rng(seed)
    return [int(rng.integers(max(-1, i - 5), i)) for i in range(n)]


TOKENS = [1, 2, 15, 16, 17, 31, 32, 33, 63, 65, 127, 128, 129, 300]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,group,page", [(64, 1, 16), (64, 8, 32), (128, 4, 16), (128, 5, 64), (256, 3, 16), (256, 16, 128)])
def test_single_tokens(dtype, dim, group, page):
    say("case tokens", dtype, dim, group, page)
    c = ref.Case(dim + group, TOKENS, [1] * len(TOKENS), dim=dim, group=group, page=page, dtype=dtype, kv_heads=1 if dim == 256 else 2)
    check_attend(c, *run_attend(c))


@pytest.mark.parametrize("softcap,bias", [(0.0, True), (6.0, False), (30.0, True)])
@pytest.mark.parametrize("dim,group,rows", [(64, 3, 5), (128, 4, 8), (256, 2, 8), (64, 4, 40), (128, 3, 50), (256, 2, 70)])
def test_trees(dim, group, rows, softcap, bias):
    """Up to 16 and 32 packed rows, and more, with sequences that consist of the tree alone."""
    say("case tree", dim, group, rows, softcap, bias)
    lens, ns = [rows, rows + 1, rows + 61, 260], [rows, rows - 1, rows, 1]
    parent = chain(rows) + [-1] * (rows - 1) + bush(rows, dim) + [-1]
    c = ref.Case(rows + dim, lens, ns, dim=dim, group=group, softcap=softcap, bias=bias, parent=parent)
    check_attend(c, *run_attend(c))


def test_the_largest_tree():
    say("case tree of 256")
    c = ref.Case(3, [700, 256], [256, 256], dim=64, group=1, kv_heads=1, parent=chain(256) + bush(256, 1), bias=True)
    check_attend(c, *run_attend(c))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,group,lens,rows", [
    (64, 1, [5, 130, 0, 257], [5, 129, 0, 257]), (128, 4, [70, 200, 33], [33, 64, 0]), (256, 2, [140, 64], [90, 64]),
    (64, 7, [100], [37]), (128, 1, [400, 1], [3, 1]), (128, 3, [900, 513, 64], [60, 130, 64]), (256, 2, [700, 333], [100, 9]),
    (64, 2, [777], [100])])
def test_chunks(dtype, dim, group, lens, rows):
    say("case chunk", dtype, dim, group, lens, rows)
    c = ref.Case(dim, lens, rows, dim=dim, group=group, dtype=dtype, bias=dim == 128, softcap=20.0 if group == 2 else 0.0)
    check_attend(c, *run_attend(c))


@pytest.mark.parametrize("rows_of", [7, 90, 200])
@pytest.mark.parametrize("with_prefix", [False, True])
def test_documents_prefix_and_rows_that_see_nothing(rows_of, with_prefix):
    """Documents that start inside and between tiles, a prefix behind a row's own slot, padding rows."""
    say("case documents", rows_of, with_prefix)
    lens, rows = [rows_of + 40, rows_of], [rows_of, rows_of]
    start = []
    for n, r in zip(lens, rows):
        start += [(n - r + i) // 33 * 33 if i % 9 else 1 << 30 for i in range(r)]
    c = ref.Case(rows_of, lens, rows, group=2, row_start=start, prefix=[45, 0] if with_prefix else None)
    out, lse = run_attend(c)
    check_attend(c, out, lse)
    z = c.attend()[1]
    assert np.isneginf(z).any() and (out.cpu()[np.isneginf(z)] == 0).all()


@pytest.mark.parametrize("rows", [3, 60])
def test_prefix_of_a_tree_stops_at_its_base(rows):
    c = ref.Case(rows, [rows + 20], [rows], group=1, parent=bush(rows), prefix=[rows + 19], row_start=[15] * rows)
    check_attend(c, *run_attend(c))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("form", ["few", "many"])
def test_what_is_not_seen_may_be_anything(dtype, form):
    """NaN and infinities in keys and values of slots that some rows see and others do not: rows that do not see them
    are as if they were not there, rows that do get what arithmetic says."""
    say("case not finite", dtype, form)
    n = 6 if form == "few" else 100
    parent = bush(n, 5)
    c = ref.Case(11, [n + 50], [n], group=2, parent=parent, dtype=dtype)
    base = 50

    def put(pool, slot, value, col):
        pool[c.table[0, slot // 16], slot % 16, :, col] = value
    put(c.v, base + 2, float("nan"), 3)
    put(c.v, base + 4, float("inf"), 7)
    put(c.v, base + 1, float("-inf"), 9)
    put(c.k, base + 5, float("nan"), 0)
    out, lse = run_attend(c)
    o, z = c.attend()
    assert np.isnan(o).any() and np.isinf(o).any() and np.isfinite(o).any()
    check_attend(c, out, lse, (o, z))
    # a document mask: the same between rows of a chunk
    start = [i // 3 * 3 for i in range(n)]
    c = ref.Case(12, [n], [n], group=2, row_start=start, dtype=dtype)
    put(c.v, 4, float("nan"), 3)
    put(c.k, 2, float("inf"), 1)
    out, lse = run_attend(c)
    o, z = c.attend()
    assert np.isnan(o).any() and np.isfinite(o).any()
    check_attend(c, out, lse, (o, z))


@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-3, 5.0])
@pytest.mark.parametrize("group,rows", [(2, 3), (4, 40)])
def test_scales(scale, group, rows):
    """Scores that are all alike, turned round, flat, and a softmax that picks single slots."""
    say("case scale", scale, group, rows)
    for softcap in (0.0, 4.0):
        c = ref.Case(rows, [300, rows], [rows, rows], dim=128, group=group, scale=scale, softcap=softcap)
        g = gpu_cache(c)
        out, lse = run_attend(c)
        check_attend(c, out, lse)
        check_weigh(c, g.weigh(c.q.cuda(), lse, ints(c.offset), ints(c.lens), **mask(c)), lse, 1.0, None)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("group,rows,n", [(2, 3, 40), (2, 3, 2500), (2, 80, 100), (2, 20, 2500)])
def test_queries_that_are_not_numbers(dim, group, rows, n):
    """A row whose query has a NaN gets NaN, its neighbours what they always get; one chunk and several."""
    c = ref.Case(n, [n], [rows], kv_heads=1, group=group, dim=dim)
    want = run_attend(c)
    c.q[1, 0, 3] = float("nan")
    out, lse = run_attend(c)
    assert out[1, 0].isnan().all() and lse[1, 0].isnan()
    keep = np.ones((rows, group), bool)
    keep[1, 0] = False
    import torch
    assert torch.equal(out[torch.from_numpy(keep)], want[0][torch.from_numpy(keep)])
    assert torch.equal(lse[torch.from_numpy(keep)], want[1][torch.from_numpy(keep)])


def test_scores_of_minus_infinity():
    """A row all of whose scores are -inf has nothing to average: zeros and -inf, like a row that sees nothing."""
    for n in (2, 80):
        c = ref.Case(5, [n], [n], group=1, kv_heads=1)
        c.q[:, :, 0], c.k[..., 0] = 1.0, float("-inf")
        out, lse = run_attend(c)
        assert (out == 0).all() and np.isneginf(lse.cpu().numpy()).all()


@pytest.mark.parametrize("rows,form", [(1, "tree"), (9, "tree"), (33, "chunk")])
def test_long_sequences_are_cut_and_joined(rows, form):
    say("case long", rows, form)
    lens = [5000, 4099, rows, 130]
    parent = sum((bush(rows) for _ in lens), []) if form == "tree" else None
    c = ref.Case(rows, lens, [rows] * 4, kv_heads=1, group=2, parent=parent)
    check_attend(c, *run_attend(c))
    # lengths far below max_len: parts of the split that have nothing
    out, lse = run_attend(c, max_len=5008)
    check_attend(c, out, lse)


def test_layouts_and_strides():
    import torch
    for layout, gap in (("heads first", 0), ("slots first", 64), ("heads first", 8)):
        for rows in (1, 45):
            c = ref.Case(gap + rows, [100, 61], [rows, rows], layout=layout, gap=gap, group=2)
            g = gpu_cache(c)
            wide = torch.full((c.q.shape[0], 9, 80), 7.0, dtype=c.dtype, device="cuda")
            q, out = wide[:, 1:5, 8:72], torch.zeros_like(wide)[:, 2:6, 16:]
            q.copy_(c.q)
            got, lse = g.attend(q, ints(c.offset), ints(c.lens), out=out, **mask(c))
            assert got is out
            check_attend(c, out, lse)


def test_offsets_past_32_bits():
    """Blocks that lie more than 2^32 elements into the pool."""
    import torch

    import paper_2605_24259_amd as rkc
    c = ref.Case(21, [150, 64], [2, 64], kv_heads=1, group=2)
    blocks, per = 70000, 16 * 4096 + 64
    assert (blocks - 20) * per > 1 << 32
    pools = []
    for x in (c.k, c.v):
        y = torch.empty_strided((blocks, 16, 1, 64), (per, 64, 64, 1), dtype=x.dtype, device="cuda")
        y[blocks - x.shape[0]:] = x.cuda()
        pools.append(y)
    g = rkc.PagedCache(*pools, (c.table + (blocks - c.k.shape[0])).to(torch.int32).cuda())
    out, lse = g.attend(c.q.cuda(), ints(c.offset), ints(c.lens), **mask(c))
    check_attend(c, out, lse)
    w = g.weigh(c.q.cuda(), lse, ints(c.offset), ints(c.lens), **mask(c))
    check_weigh(c, w, lse, 1.0, None)
    length, _, _ = g.evict(torch.rand(2, 1, 150, device="cuda"), ints(c.lens), ints([30, 30]))
    assert length.tolist() == [30, 30] and not g.status.any().item()


def check_weigh(c, w, lse, decay, weight):
    z = lse.double().cpu().numpy()
    want = c.weigh(z, decay, weight)
    got = w.double().cpu().numpy()[:, :, : want.shape[2]]
    inside = ~np.isnan(want)
    a = 2.0 ** -20 * (8 + reach(c))
    tol = a * np.nan_to_num(want) + 2.0 ** -22 * np.nan_to_num(want) + 1e-30
    assert np.all(np.abs(got - want)[inside] <= tol[inside]), np.nanmax((np.abs(got - want) / tol)[inside])
    return inside


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,group,lens,rows,kw", [
    (64, 3, [1, 17, 300], [1, 1, 1], {}), (128, 4, [40, 600], [32, 32], {}), (256, 2, [129, 70], [9, 70], dict(softcap=15.0)),
    (64, 1, [300], [300], dict(bias=True)), (128, 5, [90, 60], [60, 60], dict(tree=True, bias=True)),
    (64, 2, [200, 100], [100, 100], dict(docs=True))])
def test_weigh(dtype, dim, group, lens, rows, kw):
    say("case weigh", dtype, dim, group, lens, rows, kw)
    import torch
    kw = dict(kw)
    if kw.pop("tree", False):
        kw["parent"] = sum((bush(r, r) for r in rows), [])
    if kw.pop("docs", False):
        kw["row_start"] = [i // 30 * 30 if i % 7 else 1 << 30 for r in rows for i in range(r)]
        kw["prefix"] = [10, 0]
    c = ref.Case(dim + group, lens, rows, dim=dim, group=group, dtype=dtype, **kw)
    g = gpu_cache(c)
    q, o, n = c.q.cuda(), ints(c.offset), ints(c.lens)
    out, lse = g.attend(q, o, n, **mask(c))
    check_weigh(c, g.weigh(q, lse, o, n, **mask(c)), lse, 1.0, None)
    # onto an account, in place and not, and what lies behind the lengths stays
    w = c.weight.cuda()
    to = torch.full_like(w, 5.0)
    length = c.weight.shape[2]
    assert g.weigh(q, lse, o, n, weight=w, decay=0.5, weight_out=to, max_len=max(lens), **mask(c)) is to
    inside = check_weigh(c, to, lse, 0.5, c.weight)
    assert (to.cpu().numpy()[:, :, : max(lens)][~inside] == 5).all() and (to[:, :, max(lens):] == 5).all() and length > max(lens)
    g.weigh(q, lse, o, n, weight=w, decay=0.5, weight_out=w, max_len=max(lens), **mask(c))
    assert torch.equal(w[torch.from_numpy(np.pad(inside, ((0, 0), (0, 0), (0, length - max(lens)))))],
                       to[torch.from_numpy(np.pad(inside, ((0, 0), (0, 0), (0, length - max(lens)))))])
    # with the attention itself
    out2, lse2, w2 = g.attend(q, o, n, weight=c.weight.cuda(), decay=0.5, **mask(c, max_len=max(lens)))
    check_attend(c, out2, lse2)
    check_weigh(c, w2, lse2, 0.5, c.weight)
    assert not g.status.any().item()


@pytest.mark.parametrize("rows", [1, 2, 4, 30])
def test_account_of_documents(rows):
    """Attention with its account where slots lie before every row's document, with and without a prefix."""
    for prefix in (None, [50, 7]):
        lens = [700, 300]
        c = ref.Case(rows, lens, [rows] * 2, dim=128, group=2, row_start=[min(x, 650) for x in [400] * rows + [130] * rows], prefix=prefix)
        g = gpu_cache(c)
        w = c.weight.cuda()
        out, lse, got = g.attend(c.q.cuda(), ints(c.offset), ints(c.lens), weight=w, decay=0.5, **mask(c, max_len=700))
        check_attend(c, out, lse)
        check_weigh(c, got, lse, 0.5, c.weight)


def test_no_rows():
    """Sequences without rows: the account decays, nothing else happens."""
    import torch
    c = ref.Case(1, [20, 5], [0, 0])
    g = gpu_cache(c)
    w = c.weight.cuda()
    out, lse, w2 = g.attend(c.q.cuda(), ints(c.offset), ints(c.lens), weight=w, decay=0.25, **mask(c, max_len=20))
    assert out.shape[0] == 0 and torch.equal(w2[0, :, :20], 0.25 * w[0, :, :20]) and torch.equal(w2[1, :, :5], 0.25 * w[1, :, :5])
    assert (w2[1, :, 5:] == 0).all()


# ------------------------------------------------------------------------------------------------------------
def evict_case(seed, lens, heads=2, dim=64, page=16, dtype="bfloat16", spread="long-tailed"):
    import torch
    c = ref.Case(seed, lens, [0] * len(lens), kv_heads=heads, group=1, dim=dim, page=page, dtype=dtype)
    rng = np.random.default_rng(seed)
    n = max(lens) + 1
    w = np.exp(2 * rng.standard_normal((len(lens), heads, n)))
    if spread == "ties":
        w = rng.integers(0, 4, w.shape).astype(float)
    elif spread == "equal":
        w[:] = 0.25
    elif spread == "any":
        w *= rng.choice([1, -1, 0.0, -0.0, np.inf, -np.inf, np.nan, 1e-40], w.shape)
    pos = np.stack([[rng.permutation(2 * n)[:n] for _ in range(heads)] for _ in lens])
    return c, torch.from_numpy(w.astype(np.float32)), torch.from_numpy(pos.astype(np.int32))


def check_evict(c, w, pos, budget, protect, recent_from, **kw):
    import torch
    g = gpu_cache(c)
    k0, v0 = g.k.clone(), g.v.clone()
    n, wd = ints(c.lens), w.cuda()
    length, wo, po = g.evict(wd, n, ints(budget), protect=ints(protect), recent_from=ints(recent_from),
                             pos=None if pos is None else pos.cuda(), **kw)
    wo, po, k, v = wo.cpu(), po.cpu(), g.k.cpu(), g.v.cpu()
    k0, v0 = k0.cpu(), v0.cpu()
    k1, v1 = k0.clone(), v0.clone()
    bits = torch.int16
    for s, size in enumerate(c.lens):
        for h in range(c.kv_heads):
            p = np.arange(w.shape[2]) if pos is None else pos[s, h].numpy()
            new, src = ref.evict(w[s, h].numpy(), p, size, budget[s], 0 if protect is None else protect[s],
                                 1 << 40 if recent_from is None else recent_from[s])
            assert int(length[s]) == new
            assert torch.equal(wo[s, h, :new].view(torch.int32), w[s, h][src].view(torch.int32))
            assert po[s, h, :new].tolist() == [int(p[j]) for j in src]
            for to, j in enumerate(src):
                if to != j:
                    for x, x0 in ((k1, k0), (v1, v0)):
                        x[c.table[s, to // c.page], to % c.page, h] = x0[c.table[s, j // c.page], j % c.page, h]
    # everything that is not a gap is as it was, bit for bit
    assert torch.equal(k.contiguous().view(bits), k1.contiguous().view(bits))
    assert torch.equal(v.contiguous().view(bits), v1.contiguous().view(bits))
    assert not g.status.any().item()


@pytest.mark.parametrize("spread", ["long-tailed", "ties", "equal", "any"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (256, 32)])
def test_evict(spread, dim, page):
    say("case evict", spread, dim, page)
    lens = [1, 2, 16, 17, 100, 257, 63, 0, 90]
    c, w, pos = evict_case(dim, lens, dim=dim, page=page, spread=spread)
    n = 2 * (max(lens) + 1)
    check_evict(c, w, pos, [0, 1, 16, 5, 40, 100, 64, 3, 0], [0, 0, 3, 9, 16, 0, 70, 0, 0],
                [n, 0, 5, n, n - 200, n - 60, 0, n, 0])
    check_evict(c, w, None, [1, 1, 4, 16, 99, 256, 0, 0, 45], None, None)
    check_evict(c, w, None, [1, 1, 4, 16, 99, 256, 0, 0, 45], [-4, 1, 1, 1, 1, 1, 1, 1, 1], [0, 0, 0, 0, 0, 0, 0, 0, 0])


@pytest.mark.parametrize("lens,budget", [([16384, 16385], [8000, 8001]), ([33000, 20001], [100, 20000]), ([70001], [35000])])
@pytest.mark.parametrize("spread", ["long-tailed", "ties"])
def test_evict_long(lens, budget, spread):
    say("case evict long", lens, budget, spread)
    c, w, pos = evict_case(7, lens, heads=1, spread=spread)
    check_evict(c, w, pos, budget, [64] * len(lens), [2 * max(lens) - 100] * len(lens))


def test_evict_leaves_shared_blocks_alone():
    """Two sequences that share their first two blocks, protected in both."""
    import torch

    import paper_2605_24259_amd as rkc
    k = torch.randn(9, 16, 2, 64, device="cuda").bfloat16()
    v = torch.randn_like(k)
    table = torch.tensor([[8, 3, 1, 0], [8, 3, 5, 6]], dtype=torch.int32, device="cuda")
    g = rkc.PagedCache(k, v, table)
    k0, w = k.clone(), torch.rand(2, 2, 64, device="cuda")
    length, _, _ = g.evict(w, ints([64, 50]), ints([40, 10]), protect=ints([32, 32]))
    assert length.tolist() == [40, 32]
    for b in (8, 3, 2, 4, 7, 5, 6):
        assert torch.equal(k[b], k0[b])
    assert not torch.equal(k[1], k0[1])


@pytest.mark.parametrize("size,wrong", [(64, 3), (64, 1), (17000, 1), (17000, 700)])
def test_evict_leaves_out_moves_of_blocks_that_are_not_there(size, wrong):
    """A block id outside the pool: block 0, another sequence's, stays as it is, as do all but the sequence's other gaps."""
    import torch

    import paper_2605_24259_amd as rkc
    say("case evict wrong block", size, wrong)
    pages = -(-size // 16)
    k = torch.randn(pages + 1, 16, 1, 64, device="cuda").bfloat16()
    v = torch.randn_like(k)
    table = torch.arange(1, pages + 1, dtype=torch.int32, device="cuda")[None].contiguous()
    table[0, wrong] = 1 << 30
    g = rkc.PagedCache(k, v, table)
    k0, v0 = k.clone(), v.clone()
    w = torch.arange(pages * 16, dtype=torch.float32, device="cuda").view(1, 1, -1).contiguous()  # the last half stays
    length, wo, _ = g.evict(w, ints([size]), ints([size // 2]))
    new = size // 2
    assert length.tolist() == [new] and g.status.tolist() == [rkc.cache.CS_BLOCK]
    assert torch.equal(wo[0, 0, :new], w[0, 0, size - new:size])
    for x, x0 in ((k, k0), (v, v0)):
        want = x0.clone()
        flat, flat0 = want[1:].view(-1, 1, 64), x0[1:].view(-1, 1, 64)
        to = torch.arange(new, device="cuda")
        at = to + size - new
        fine = (to // 16 != wrong) & (at // 16 != wrong)
        flat[to[fine]] = flat0[at[fine]]
        assert torch.equal(x, want)


# ------------------------------------------------------------------------------------------------------------
def test_other_streams_and_repeated_calls():
    """On a side stream behind work of its own; every call gives the same bits."""
    import torch
    for rows in (1, 60):
        c = ref.Case(rows, [900, 300], [rows, rows], group=2)
        g = gpu_cache(c)
        q, o, n = c.q.cuda(), ints(c.offset), ints(c.lens)
        first = g.attend(q, o, n, weight=c.weight.cuda(), **mask(c, max_len=900))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            x = torch.randn(2048, 2048, device="cuda")
            for _ in range(5):
                x = x @ x * 1e-2
            q2 = q + (x[0, 0] * 0).nan_to_num().to(q.dtype)
        m = mask(c, max_len=900)
        side.wait_stream(torch.cuda.current_stream())
        again = [g.attend(q2, o, n, weight=c.weight.cuda(), stream=side, **m) for _ in range(3)]
        torch.cuda.synchronize()
        for r in again:
            assert all(torch.equal(a, b) for a, b in zip(first, r))


def test_in_a_graph():
    """Captured once, replayed with eager work between the replays, on inputs that change in place."""
    import torch
    c = ref.Case(2, [500, 90], [1, 1], group=4)
    g = gpu_cache(c)
    q, o, n, m = c.q.cuda(), ints(c.offset), ints(c.lens), mask(c, max_len=512)
    w, budget = torch.rand(2, 2, 512, device="cuda"), ints([200, 50])
    g.attend(q, o, n, weight=w, **m)
    g.evict(w, n, budget)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    k0, v0 = g.k.clone(), g.v.clone()
    with torch.cuda.graph(graph):
        out, lse, w1 = g.attend(q, o, n, weight=w, **m)
        length, w2, pos = g.evict(w1, n, budget)
    for turn in range(4):
        q.copy_(torch.randn_like(q))
        g.k.copy_(k0), g.v.copy_(v0)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, lse, w1, length, w2[0, :, :200], pos[0, :, :200], g.k, g.v)]
        g.k.copy_(k0), g.v.copy_(v0)
        eo, el, ew = g.attend(q, o, n, weight=w, **m)
        e = g.evict(ew, n, budget)
        want = (eo, el, ew, e[0], e[1][0, :, :200], e[2][0, :, :200], g.k, g.v)
        for a, b in zip(got, want):
            assert torch.equal(a.nan_to_num(7), b.nan_to_num(7))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,rows", [(64, 1), (128, 5), (256, 3)])
@pytest.mark.parametrize("n", [700, 5000])
def test_weights_of_few_rows_keep_their_bits(dtype, dim, rows, n):
    """Up to 16 packed rows: weights are the sum of two numbers of the type, whose error is u^2 in place of u, and for
    float16 at least half a step of 2^-24 of weights whose sum is at least 2^-2; what is left of u is the result's rounding."""
    say("case weights of few rows", dtype, dim, rows, n)
    c = ref.Case(dim + rows + n, [n, n // 3], [rows] * 2, group=3, dim=dim, dtype=dtype)
    g = gpu_cache(c)
    out, lse = g.attend(c.q.cuda(), ints(c.offset), ints(c.lens), **mask(c))
    want, z = c.attend()
    got, u = out.double().cpu().numpy(), UNIT[dtype]
    most = float(np.nan_to_num(c.v.double().numpy(), nan=0, posinf=0, neginf=0).__abs__().max())
    few = n * 2.0 ** -23 if dtype == "float16" else 0
    near = u * np.abs(want) + (2 * u * u + 2.0 ** -20 * (8 + reach(c)) + few) * most
    assert (np.abs(got - want) <= near).all()


def test_what_only_the_device_sees_is_flagged():
    """Bad lengths, row counts, block ids and parents: nothing outside the buffers is touched, the status says so and
    the other sequences are as always."""
    import torch

    import paper_2605_24259_amd as rkc
    for rows in (2, 60):
        c = ref.Case(4, [100, 100, 100, 100, 100], [rows] * 5, group=1, parent=bush(rows) * 5)
        g = gpu_cache(c)
        q, o, w = c.q.cuda(), ints(c.offset), c.weight.cuda()
        lens, parent = ints(c.lens), ints(c.parent)
        want = g.attend(q, o, lens, **mask(c))
        lens[0], lens[1] = 1 << 30, rows - 1
        parent[2 * rows + 1] = 1
        g.block_table[3, 2] = 1 << 30
        m = mask(c, parent=parent)
        out, lse = g.attend(q, o, lens, **m)
        assert g.status.tolist() == [rkc.cache.CS_LENGTH, rkc.cache.CS_LENGTH, rkc.cache.CS_PARENT, rkc.cache.CS_BLOCK, 0]
        assert torch.equal(out[4 * rows:], want[0][4 * rows:]) and torch.equal(lse[4 * rows:], want[1][4 * rows:])
        g.weigh(q, want[1], o, lens, **m)
        g.status.zero_()
        lens[2] = -1
        length, _, _ = g.evict(w, lens, ints([20] * 5))
        assert g.status.tolist()[:3] == [1, 0, 1] and length[4].item() == 20


def test_refusals():
    import torch

    import paper_2605_24259_amd as rkc
    c = ref.Case(0, [40, 20], [2, 2])
    g = gpu_cache(c)
    q, o, n, m = c.q.cuda(), ints(c.offset), ints(c.lens), mask(c)
    bad = [dict(q=q.float()), dict(q=q[:, :5]), dict(q=q[..., :32]), dict(q=q.cpu()), dict(row_offset=o[:2]), dict(row_offset=o.long()),
           dict(length=n.cpu()), dict(length=n[:1]), dict(parent=ints([-1])), dict(slope=torch.ones(3, device="cuda")), dict(prefix=ints([1])),
           dict(row_start=ints([0, 0, 0])), dict(out=torch.zeros(4, 6, 32, device="cuda")), dict(weight=torch.zeros(2, 2, 5, device="cuda"))]
    for b in bad:
        a = dict(dict(m, q=q, row_offset=o, length=n), **b)
        with pytest.raises(ValueError):
            g.attend(a.pop("q"), a.pop("row_offset"), a.pop("length"), **a)
    for b, status in ((dict(max_rows=-1), -3), (dict(max_len=1 << 20), -3), (dict(softcap=-1.0), -3), (dict(softcap=float("nan")), -3),
                      (dict(scale=float("nan")), -3), (dict(parent=ints([-1] * 4), max_rows=257), -4)):
        with pytest.raises(rkc.RkcError) as e:
            g.attend(q, o, n, **dict(m, **b))
        assert e.value.status == status
    with pytest.raises(rkc.RkcError):
        w = torch.zeros(2, 2, 40, device="cuda")
        g.evict(w, n, n, weight_out=w)
    with pytest.raises(ValueError):
        g.evict(torch.zeros(2, 3, 40, device="cuda"), n, n)
    for k in (torch.zeros(4, 16, 2, 64), torch.zeros(4, 16, 64, device="cuda").bfloat16(), torch.zeros(4, 16, 2, 64, device="cuda")):
        with pytest.raises((ValueError, TypeError)):
            rkc.PagedCache(k, k, torch.zeros(1, 4, dtype=torch.int32, device="cuda"))
    with pytest.raises(rkc.RkcError):  # 24 slots a block
        k = torch.zeros(4, 24, 2, 64, device="cuda").bfloat16()
        rkc.PagedCache(k, k, torch.zeros(2, 4, dtype=torch.int32, device="cuda")).attend(q, o, n, **m)


@pytest.mark.parametrize("softcap", [40.0, 1e3, 1e6])
@pytest.mark.parametrize("lens,rows,group", [([900, 40], [1, 1], 4), ([300, 90], [60, 33], 3), ([500, 300], [300, 140], 2)])
def test_cap_far_above_the_scores(lens, rows, group, softcap):
    """A cap that the scores do not come near changes them by a relative error, not by one of the cap's size: the
    tolerance of an uncapped score, relative to |scale| |q| |k| alone (the cap's own form: 2 units of 2^-24 of a score
    in place of the 16 that 2^-20 stands for)."""
    import torch
    say("case cap", lens, rows, group, softcap)
    c = ref.Case(11, lens, rows, dim=128, group=group, softcap=softcap)
    o, z = c.attend()
    out, lse = run_attend(c)
    a = 2.0 ** -20 * (8 + reach(c) - softcap)
    assert np.abs(lse.double().cpu().numpy() - z).max() <= a
    u, vmax = UNIT["bfloat16"], np.nan_to_num(np.abs(c.v.double().numpy()), nan=0, posinf=0).max()
    assert np.all(np.abs(out.double().cpu().numpy() - o) <= u * (vmax + np.abs(o)) + a * vmax)
    w = gpu_cache(c).weigh(c.q.cuda(), torch.from_numpy(z).float().cuda(), ints(c.offset), ints(c.lens), **mask(c)).double().cpu().numpy()
    want = c.weigh(z, 1.0)
    for s, n in enumerate(lens):  # the sums of the softmax, given in 32 bits, have an error of 2^-24 of theirs
        assert np.all(np.abs(w[s, :, :n] - want[s, :, :n]) <= (a + 2.0 ** -23 * np.abs(z).max()) * want[s, :, :n] + 1e-30)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows", [1, 40, 300])
def test_many_small_weights(dim, rows):
    """One slot of weight 1 and 60,000 of exp(-14.5), whose float16 would have three bits left: they make up a thirtieth
    of the sum, and are as exact as all weights are: u each for the weight, the result, and half for what is below."""
    import torch

    import paper_2605_24259_amd as rkc
    say("case many small weights", dim, rows)
    n, page = 60000 + rows, 64
    pages = -(-n // page)
    k = torch.zeros(pages, page, 1, dim, dtype=torch.float16, device="cuda")
    v = torch.ones_like(k)
    k[..., 0] = -14.5
    k[0, 0], v[0, 0] = 0, 0
    q = torch.zeros(rows, 1, dim, dtype=torch.float16, device="cuda")
    q[..., 0] = 1
    g = rkc.PagedCache(k, v, torch.arange(pages, dtype=torch.int32, device="cuda")[None])
    out, _ = g.attend(q, ints([0, rows]), ints([n]), max_rows=rows, scale=1.0)
    tail = (n - rows + np.arange(rows)) * np.exp(-14.5)
    want = (tail / (1 + tail))[:, None, None]
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= 2.5 * 2.0 ** -11 * want)
