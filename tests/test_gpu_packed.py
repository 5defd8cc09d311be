"""Attention over a cache of 4 bits against the plain 64-bit implementation, on the values that the bits stand for.
Tolerances as in test_gpu_cache.py: the products are of the values themselves, which 16 bits hold exactly."""
import numpy as np
import pytest

from tests import packed_reference as ref
from tests.gpu_util import say
from tests.test_gpu_cache import TOKENS, bush, chain, check_attend, ints, mask

pytestmark = pytest.mark.gpu


def packed_cache(c, dev="cuda"):
    import paper_2605_24259_amd as rkc
    return rkc.PackedCache(c.pool.to(dev), c.table.to(dev), page_tokens=c.page, head_dim=c.dim, dtype=c.dtype)


def run_attend(c, **kw):
    g = packed_cache(c)
    r = g.attend(c.q.cuda(), ints(c.offset), ints(c.lens), **mask(c, **kw))
    assert not g.status.any().item()
    return r


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,group,page", [(64, 1, 16), (64, 8, 32), (128, 4, 16), (128, 5, 64), (256, 3, 16), (256, 16, 128)])
def test_single_tokens(dtype, dim, group, page):
    say("case tokens", dtype, dim, group, page)
    c = ref.Packed(dim + group, TOKENS, [1] * len(TOKENS), dim=dim, group=group, page=page, dtype=dtype, kv_heads=1 if dim == 256 else 2)
    check_attend(c, *run_attend(c))


@pytest.mark.parametrize("softcap,bias", [(0.0, True), (6.0, False), (30.0, True)])
@pytest.mark.parametrize("dim,group,rows", [(64, 3, 5), (128, 4, 4), (256, 2, 8), (64, 4, 40), (128, 3, 50), (256, 2, 70)])
def test_trees(dim, group, rows, softcap, bias):
    say("case tree", dim, group, rows, softcap, bias)
    lens, ns = [rows, rows + 1, rows + 61, 260], [rows, rows - 1, rows, 1]
    parent = chain(rows) + [-1] * (rows - 1) + bush(rows, dim) + [-1]
    c = ref.Packed(rows + dim, lens, ns, dim=dim, group=group, softcap=softcap, bias=bias, parent=parent)
    check_attend(c, *run_attend(c))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,group,lens,rows", [
    (64, 1, [5, 130, 0, 257], [5, 129, 0, 257]), (128, 4, [70, 200, 33], [33, 64, 0]), (256, 2, [140, 64], [90, 64]),
    (64, 7, [100], [37]), (128, 1, [400, 1], [3, 1]), (128, 3, [900, 513, 64], [60, 130, 64]), (256, 2, [700, 333], [100, 9]),
    (64, 2, [777], [100]), (128, 2, [600, 580], [400, 300])])
def test_chunks(dtype, dim, group, lens, rows):
    say("case chunk", dtype, dim, group, lens, rows)
    c = ref.Packed(dim, lens, rows, dim=dim, group=group, dtype=dtype, bias=dim == 128, softcap=20.0 if group == 2 else 0.0)
    check_attend(c, *run_attend(c))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("rows_of", [7, 90, 200])
@pytest.mark.parametrize("with_prefix", [False, True])
def test_documents_prefix_and_rows_that_see_nothing(rows_of, with_prefix, dim):
    say("case documents", rows_of, with_prefix, dim)
    lens, rows = [rows_of + 40, rows_of], [rows_of, rows_of]
    start = []
    for n, r in zip(lens, rows):
        start += [(n - r + i) // 33 * 33 if i % 9 else 1 << 30 for i in range(r)]
    c = ref.Packed(rows_of, lens, rows, group=2, dim=dim, row_start=start, prefix=[45, 0] if with_prefix else None)
    out, lse = run_attend(c)
    check_attend(c, out, lse)
    if not with_prefix:
        nothing = ints(start).eq(1 << 30)
        assert nothing.any() and out[nothing].eq(0).all() and lse[nothing].eq(float("-inf")).all()


@pytest.mark.parametrize("dim,group,rows,dtype", [(64, 1, 3, "float16"), (128, 4, 4, "bfloat16"), (256, 2, 6, "bfloat16"),
                                                  (64, 3, 30, "bfloat16"), (128, 2, 100, "float16"), (256, 1, 90, "float16")])
def test_marked_slots_reach_the_rows_that_see_them(dim, group, rows, dtype):
    """A marked slot before all rows, between them, and (for documents) out of sight of some."""
    say("case marks", dim, group, rows, dtype)
    n = 200
    start = [120 if i % 2 else 0 for i in range(rows)]
    c = ref.Packed(dim, [n, n], [rows, rows], dim=dim, group=group, dtype=dtype, row_start=start + [0] * rows,
                   marks=[(0, 50, 0), (1, n - rows + 1, 1)])
    out, lse = run_attend(c)
    check_attend(c, out, lse)
    got = lse.isnan().cpu().numpy()
    assert got[:rows:2, :group].all() and not got[1:rows:2].any() and not got[:rows, group:].any()
    assert not got[rows, :].any() and got[rows + 1:, group:].all() and not got[rows:, :group].any()


@pytest.mark.parametrize("rows,group,dim", [(1, 4, 128), (3, 1, 64), (1, 2, 256), (40, 4, 128), (100, 1, 256), (64, 2, 64)])
def test_long_sequences_in_parts(rows, group, dim):
    say("case parts", rows, group, dim)
    c = ref.Packed(rows, [9000, 17, 4100], [rows, min(rows, 17), rows], group=group, dim=dim, kv_heads=1, page=64)
    check_attend(c, *run_attend(c))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("group,rows,form", [(1, 20, "tree"), (1, 32, "tree"), (3, 11, "tree"), (2, 32, "tree"), (4, 24, "tree"), (1, 33, "tree"),
                                             (3, 31, "chunk"), (1, 90, "chunk"), (1, 33, "chunk"), (2, 20, "documents"), (3, 32, "documents"),
                                             (17, 1, "chunk"), (48, 2, "tree"), (1, 97, "chunk")])
def test_middling_rows(dim, group, rows, form):
    """One and more tiles of 32 packed rows, the last one in part, sequences of fewer rows and tiles beside them."""
    say("case middling", dim, group, rows, form)
    lens, ns = [rows, rows + 13, 2 * rows + 700, 5, 0, 1500], [rows, rows, rows // 2, min(rows, 5), 0, 1]
    kw = {}
    if form == "tree":
        kw = dict(parent=sum((bush(n, n + dim) for n in ns), []), bias=rows % 2 == 0)
    elif form == "documents":
        kw = dict(row_start=[(n - r + i) // 33 * 33 if i % 9 else 1 << 30 for n, r in zip(lens, ns) for i in range(r)], prefix=[15, 0, 40, 0, 0, 0])
    else:
        kw = dict(bias=rows % 2 == 1)
    c = ref.Packed(rows + dim, lens, ns, dim=dim, group=group, kv_heads=2, dtype="float16" if group % 2 else "bfloat16",
                   softcap=15.0 if rows == 32 else 0.0, **kw)
    out, lse = run_attend(c)
    check_attend(c, out, lse, want=c.attend_at_once())


@pytest.mark.parametrize("dim,seqs,longest", [(64, 33, 1100), (128, 33, 300), (64, 3, 1300), (128, 61, 40), (64, 70, 100)])
def test_many_sequences(dim, seqs, longest):
    """Of unlike lengths, whole and in parts, in the order of their lengths and not; equal ones and empty ones among them."""
    say("case sequences", dim, seqs, longest)
    rng = np.random.default_rng(dim + seqs)
    lens = [int(x) for x in rng.integers(1, longest, seqs)]
    lens[:3], lens[-1] = [longest, 1, lens[-1]], longest
    rows = [1] * seqs
    if seqs > 5:
        lens[4], rows[4] = 0, 0
    c = ref.Packed(seqs, lens, rows, dim=dim, group=2, kv_heads=16, page=64)
    check_attend(c, *run_attend(c, max_len=longest), want=c.attend_at_once())


LONG = [  # dim, dtype, group, lens, rows, what else: more than 128 packed rows, row tiles x parts of 256 slots past 512
    (128, "bfloat16", 4, [7000, 6001], [300, 257], {}), (128, "float16", 4, [7000, 6001], [300, 257], dict(softcap=20.0)),
    (128, "bfloat16", 4, [7000, 6001], [300, 257], dict(softcap=300.0, bias=True)), (128, "float16", 2, [9000, 70], [600, 70], dict(bias=True)),
    (256, "bfloat16", 4, [7000, 6001], [300, 257], {}), (256, "float16", 4, [7000, 6001], [300, 257], dict(softcap=30.0)),
    (256, "bfloat16", 2, [9000, 70], [600, 70], dict(bias=True)), (128, "bfloat16", 5, [8192, 8000, 30, 5000], [64, 50, 30, 1], "tree"),
    (256, "float16", 5, [8192, 8000, 30, 5000], [64, 50, 30, 1], "tree"), (128, "bfloat16", 4, [7000, 6001], [700, 500], "documents"),
    (256, "bfloat16", 4, [7000, 6001], [700, 500], "documents"), (64, "bfloat16", 4, [7000, 6001], [300, 257], dict(softcap=20.0)),
    (128, "bfloat16", 32, [5000, 900, 64, 1], [8, 8, 8, 1], "tree"), (128, "float16", 8, [20000, 3, 12000], [30, 3, 20], {}),
    (256, "bfloat16", 8, [20000, 3, 12000], [12, 3, 16], {}), (64, "float16", 8, [20000, 3, 12000], [30, 3, 20], {})]


@pytest.mark.parametrize("case", LONG)
def test_many_rows_of_long_sequences(case):
    """Both sizes of a workgroup, whole and cut sequences, short ones beside them."""
    dim, dtype, group, lens, rows, what = case
    say("case long", *case)
    kw = dict(what) if isinstance(what, dict) else {}
    if what == "tree":
        kw = dict(parent=sum((bush(r, dim + r) for r in rows), []), bias=True)
    elif what == "documents":
        start = [x for n, r in zip(lens, rows) for x in [(n - r + i) // 333 * 333 if i % 9 else 1 << 30 for i in range(r)]]
        kw = dict(row_start=start, prefix=[1000, 0])
    c = ref.Packed(len(lens) + dim, lens, rows, dim=dim, group=group, dtype=dtype, page=64, **kw)
    check_attend(c, *run_attend(c), want=c.attend_at_once())


def test_strides_of_the_pool_and_of_rows():
    """A slice of a pool's heads, blocks apart, queries of a fused tensor and outputs among others."""
    import torch

    import paper_2605_24259_amd as rkc
    say("case strides")
    c = ref.Packed(5, [70, 41], [5, 41], group=2, dim=64)
    n = c.pool.shape[2]
    wide = torch.randint(0, 256, (c.pool.shape[0], 5, n + 48), dtype=torch.uint8).cuda()
    wide[:, 1:3, 16:n + 16] = c.pool.cuda()
    g = rkc.PackedCache(wide[:, 1:3, 16:n + 16], c.table.cuda(), page_tokens=c.page, head_dim=64, dtype=c.dtype)
    q = torch.zeros(46, 7, 64, dtype=c.dtype, device="cuda")
    q[:, 2:6] = c.q.cuda()
    out = torch.full((46, 6, 128), 2.0, dtype=c.dtype, device="cuda")
    got, lse = g.attend(q[:, 2:6], ints(c.offset), ints(c.lens), out=out[:, 1:5, 64:], **mask(c))
    check_attend(c, got, lse)
    assert got.data_ptr() == out[:, 1:5, 64:].data_ptr() and out[..., :64].eq(2).all() and out[:, 0].eq(2).all() and out[:, 5].eq(2).all()
    # in the place of the queries
    again, _ = g.attend(q[:, 2:6], ints(c.offset), ints(c.lens), out=q[:, 2:6], **mask(c))
    assert torch.equal(again, got)
    # and the slice's slots can be written: its neighbours stay
    x = torch.randn(46, 2, 64, device="cuda").to(c.dtype)
    before = wide.clone()
    g.store(x, x, ints(c.offset), ints(c.lens))
    assert wide[:, 0].equal(before[:, 0]) and wide[:, 3:].equal(before[:, 3:]) and wide[..., :16].equal(before[..., :16])
    assert wide[..., n + 16:].equal(before[..., n + 16:])


def test_bad_lengths_blocks_and_parents():
    """Told of, and nothing outside is read; sequences that are fine keep their results."""
    import torch
    say("case bad")
    for rows in (3, 40):
        c = ref.Packed(rows, [80, 90, 100, 60], [rows] * 4, group=2, dim=64, parent=(chain(rows) * 4))
        g = packed_cache(c)
        lens, parent = list(c.lens), list(c.parent)
        lens[0] = 1 << 25
        g.block_table[1, 2] = -5
        parent[2 * rows + 1] = rows
        out = torch.full_like(c.q, 9.0).cuda()
        got, lse = g.attend(c.q.cuda(), ints(c.offset), ints(lens), out=out, **dict(mask(c), parent=ints(parent)))
        assert g.status.tolist() == [1, 2, 4, 0]
        assert got[:rows].eq(9).all()
        o, z = c.attend()
        assert np.abs(lse[3 * rows:].cpu().numpy() - z[3 * rows:]).max() < 1e-3
        # of the second, block 0 was read in part, which nobody owns here or somebody else does: anything
        assert got[2 * rows:].isfinite().all() and lse[2 * rows:].isfinite().all()


def test_twice_the_same_and_captured():
    """No sum goes by the order of workgroups; replays give the same among other work, two graphs beside each other."""
    import torch
    say("case graph")
    cases = [ref.Packed(1, [9000, 300, 77], [1, 1, 1], group=4, dim=128, kv_heads=1), ref.Packed(2, [5000, 300], [40, 40], group=4, dim=128, kv_heads=1)]
    runs = []
    for c in cases:
        g, q, off, lens, m = packed_cache(c), c.q.cuda(), ints(c.offset), ints(c.lens), mask(c)
        want = g.attend(q, off, lens, **m)
        for _ in range(3):
            got = g.attend(q, off, lens, **m)
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        other = torch.cuda.Stream()
        got = g.attend(q, off, lens, stream=other, **m)
        other.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = g.attend(q, off, lens, **m)
        runs.append((graph, out, want, g, q, off, lens, m))
    for turn in range(4):
        for graph, out, want, g, q, off, lens, m in runs:
            for x in out:
                x.zero_()
        for graph, *_ in runs:
            graph.replay()
        eager = runs[turn % 2][3].attend(*runs[turn % 2][4:7], **runs[turn % 2][7])
        torch.cuda.synchronize()
        for graph, out, want, *_ in runs:
            assert all(torch.equal(a, b) for a, b in zip(out, want)), turn
        assert all(torch.equal(a, b) for a, b in zip(eager, runs[turn % 2][2]))


def test_refusals():
    import torch

    import paper_2605_24259_amd as rkc
    c = ref.Packed(1, [40, 20], [2, 1], group=2, dim=64)
    g, q, off, lens = packed_cache(c), c.q.cuda(), ints(c.offset), ints(c.lens)
    for args, kw in (((q[..., :32], off, lens), {}), ((q.float(), off, lens), {}), ((q[:, :3], off, lens), {}), ((q, off[:1], lens), {}),
                     ((q, off, lens.long()), {}), ((q, off, lens), dict(slope=torch.ones(3, device="cuda"))), ((q, off, lens), dict(out=q[:1])),
                     ((q, off, lens), dict(parent=ints([0])))):
        with pytest.raises(ValueError):
            g.attend(*args, max_rows=2, **kw)
    for kw in (dict(softcap=-1.0), dict(max_len=1 << 20), dict(parent=ints([-1, 0, -1]), max_rows=300), dict(out=q[:1].expand(3, -1, -1))):
        with pytest.raises(rkc.RkcError):
            g.attend(q, off, lens, **dict(dict(max_rows=2), **kw))
    assert not hasattr(g, "weigh") and not hasattr(g, "evict")


def test_a_claim_in_four_bits():
    """The operators as they are used together: a prompt's rows are normed, turned and stored in 16 bits; the claim is demoted
    to 4 bits, block by block of its rows, attended to with drafted tokens and by a decode step whose token is stored in the
    same pass, and brought back to 16 bits."""
    import torch

    import paper_2605_24259_amd as rkc
    say("case claim")
    g = torch.Generator(device="cuda").manual_seed(4)
    f, n, drafts, H, G, D, page = torch.bfloat16, 300, 6, 2, 4, 128, 16

    def rand(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(f)
    pages = 24
    table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)[None]
    paged = rkc.PagedCache(torch.zeros(pages, page, H, D, dtype=f, device="cuda"), torch.zeros(pages, page, H, D, dtype=f, device="cuda"), table)
    packed = rkc.PackedCache(rkc.PackedCache.pool(pages, page, H, D), table.flip(1).contiguous(), page_tokens=page, head_dim=D, dtype=f)
    turn = dict(freq=(1e4 ** (-torch.arange(D // 2, device="cuda") * 2 / D)).float(), k_norm=1 + 0.1 * torch.randn(D, generator=g, device="cuda"))
    q_norm = 1 + 0.1 * torch.randn(D, generator=g, device="cuda")
    whole = ints([0, n]), ints([n])
    x = rand(n, (G + 2) * H, D)
    q = paged.store(x[:, -2 * H: -H], x[:, -H:], *whole, q=x[:, : G * H], q_norm=q_norm, **turn)
    out16, lse16 = paged.attend(q, *whole, max_rows=n)
    k, v = paged.read(*whole, rows=n)
    packed.store(k, v, *whole)  # demoted: as they are, normed and turned before
    back = packed.read(*whole, rows=n)
    want = [torch.from_numpy(ref.held(t.float().cpu().numpy(), "bfloat16")[2]).to(f).cuda() for t in (k, v)]
    assert all(torch.equal(a, b) for a, b in zip(back, want))
    # 4 bits are off by at most a sixth of the value, or a quarter of the smallest step: outputs stay near the others
    out, lse = packed.attend(q, *whole, max_rows=n)
    assert 0.5 < torch.nn.functional.cosine_similarity(out.float().flatten(), out16.float().flatten(), dim=0)
    # drafted tokens behind it
    parent = [-1, 0, 0, 1, 1, 2]
    y = rand(drafts, (G + 2) * H, D)
    pos = ints([n + d for d in (0, 1, 1, 2, 2, 2)])
    tree = ints([0, drafts]), ints([n + drafts])
    qd = packed.store(y[:, -2 * H: -H], y[:, -H:], *tree, q=y[:, : G * H], q_norm=q_norm, position=pos, **turn)
    out, lse = packed.attend(qd, *tree, max_rows=drafts, parent=ints(parent))
    kk, vv = packed.read(ints([0, n + drafts]), ints([n + drafts]), rows=n + drafts)
    assert torch.equal(kk[:n], back[0]) and torch.equal(vv[:n], back[1])
    lines = []
    for p in parent:
        lines.append((lines[p] if p >= 0 else []) + [len(lines)])
    vmax = float(vv.abs().max())
    for i, line in enumerate(lines):
        at = list(range(n)) + [n + j for j in line]
        for h in range(H * G):
            s = kk[at, h // G].double().cpu() @ qd[i, h].double().cpu() / D ** 0.5
            want = torch.softmax(s, 0) @ vv[at, h // G].double().cpu()
            assert (out[i, h].double().cpu() - want).abs().max() <= 2.0 ** -8 * 2 * vmax  # weights and outputs rounded to bfloat16
            assert abs(float(lse[i, h]) - float(torch.logsumexp(s, 0))) < 2.0 ** -12
    # the root alone, stored and attended to again as a single token: the same bits as its row of the tree were stored with
    one = ints([0, 1]), ints([n + 1])
    q1 = packed.store(y[:1, -2 * H: -H], y[:1, -H:], *one, q=y[:1, : G * H], q_norm=q_norm, **turn)
    assert torch.equal(q1, qd[:1]) and torch.equal(packed.read(*one, rows=1)[0], kk[n: n + 1])
    out1, lse1 = packed.attend(q1, *one, max_rows=1)
    assert (out1.double() - out[:1].double()).abs().max() <= 2.0 ** -8 * 2 * vmax and (lse1 - lse[:1]).abs().max() < 2.0 ** -12
    # brought back
    k, v = packed.read(*whole, rows=n)
    paged.store(k, v, *whole)
    assert all(torch.equal(a, b) for a, b in zip(paged.read(*whole, rows=n), back))
    assert not packed.status.any().item() and not paged.status.any().item()
