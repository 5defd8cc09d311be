"""Rows stored and read: what they tell of, what a bad block reads, rows at the ends of their types.  Tolerances as in test_gpu_rows.py."""
import numpy as np
import pytest
import torch

from tests import packed_reference as ref
from tests.gpu_util import say
from tests.test_gpu_cache import ints
from tests.test_gpu_rows import Rows, bits

pytestmark = pytest.mark.gpu


def contents(r, kind):
    """Clones of what a cache holds."""
    return [x.clone() for x in ((r.cache.k, r.cache.v) if kind == "cache" else (r.packed.pool,))]


@pytest.mark.parametrize("kind", ["cache", "packed"])
@pytest.mark.parametrize("offset,lens,told", [
    ([0, 5, 3, 14, 14], [5, 5, 11, 0], [0, 1, 0, 0]),           # back: rows 3 and 4 belong to one of two sequences
    ([0, 5, 5, 3, 14], [5, 5, 5, 14], [0, 0, 1, 0]),
    ([0, 14, 14, 14, 14], [14, -1, 1 << 20, 0], [0, 1, 1, 0]),  # lengths of sequences without rows
    ([-2, 3, 3, 14, 14], [30, 3, 11, 2], [1, 0, 0, 0]),
    ([0, 3, 3, 12, 15], [3, 3, 9, 20], [0, 0, 0, 1]),           # more rows than there are
    ([2, 4, 2, 9, 14], [2, 0, 9, 5], [0, 1, 0, 0])])
def test_sequences_are_told_of(kind, offset, lens, told):
    """As attention tells of them, whether a row leads to them or not; what is fine is stored, nothing else is written."""
    say("case told", kind, offset, lens)
    r = Rows(9, [2, 3, 4, 5], [20, 1, 0, 30], norm=None, rot=0)
    c, before = getattr(r, kind), contents(r, kind)
    c.store(r.k, r.v, ints(offset), ints(lens))
    assert c.status.tolist() == told
    c.status.zero_()
    k, v = (torch.full((14, 2, 128), 5.0, dtype=r.dtype, device="cuda") for _ in range(2))
    c.read(ints(offset), ints(lens), rows=14, k=k, v=v)
    assert c.status.tolist() == told
    if kind == "packed":
        c.status.zero_()
        c.attend(r.q[:, :2].contiguous(), ints(offset), ints(lens), max_rows=14)
        assert c.status.tolist() == told
    # slots that some sequence's rows may have, and those that only one has
    slots, rows = {}, {}
    for s in range(4):
        if not told[s]:
            for t in range(offset[s], offset[s + 1]):
                j = lens[s] - (offset[s + 1] - t)
                slots.setdefault((int(r.table[s, j // 16]), j % 16), []).append(t)
                rows.setdefault(t, []).append((int(r.table[s, j // 16]), j % 16))
    for t in range(14):
        if t not in rows:  # left alone
            assert k[t].eq(5).all() and v[t].eq(5).all()
        elif kind == "cache":
            assert any(bits(c.k[at].contiguous()).equal(bits(r.k[t].contiguous())) for at in rows[t]) and bits(v[t].contiguous()).equal(bits(r.v[t].contiguous()))
        else:
            for got, x in ((k, r.k), (v, r.v)):
                assert got[t].equal(torch.from_numpy(ref.held(x[t].float().cpu().numpy(), r.name)[2]).to(r.dtype).cuda())
    mine = torch.zeros(c._c.n_blocks, 16, dtype=torch.bool)
    for at in slots:
        mine[at] = True
    mine = mine.cuda()
    now = contents(r, kind)
    if kind == "cache":
        for x, y in zip(now, before):
            assert bits(x)[~mine].equal(bits(y)[~mine])
    else:
        for x, y in zip(ref.split(now[0].cpu().numpy(), 16, 128), ref.split(before[0].cpu().numpy(), 16, 128)):
            x, y = x.swapaxes(1, 2), y.swapaxes(1, 2)
            assert np.array_equal(x[~mine.cpu().numpy()], y[~mine.cpu().numpy()])


@pytest.mark.parametrize("seqs,bad", [(5000, (0, 63, 64, 700, 4999)), (200, (199,)), (300000, (0, 150000, 299999))])
def test_many_sequences_without_rows_are_told_of(seqs, bad):
    say("case many told", seqs)
    import paper_2605_24259_amd as rkc
    c = rkc.PackedCache(rkc.PackedCache.pool(2, 16, 1, 64), torch.zeros(seqs, 1, dtype=torch.int32, device="cuda"), page_tokens=16, head_dim=64, dtype=torch.float16)
    lens = np.zeros(seqs, int)
    lens[list(bad)] = 17
    x = torch.zeros(3, 1, 64, dtype=torch.float16, device="cuda")
    for call in (lambda *at: c.store(x, x, *at), lambda *at: c.read(*at, rows=3)):
        call(ints(np.zeros(seqs + 1)), ints(lens))
        assert c.status.nonzero().flatten().tolist() == list(bad) and c.status.max().item() == 1
        c.status.zero_()


@pytest.mark.parametrize("kind", ["cache", "packed"])
def test_a_bad_block_reads_block_0(kind):
    """Slots of a block id outside the pool read those of block 0; the sequence's other slots read their own."""
    say("case block 0", kind)
    r = Rows(9, [0, 0, 0, 5], [20, 4, 9, 30], norm=None, rot=0)
    c = getattr(r, kind)
    x, y = (torch.randn(4, 2, 128, device="cuda").to(r.dtype) for _ in range(2))
    table = r.table.clone()
    table[0, 0], table[3] = 0, ints([5, 6, 7])
    c.block_table.copy_(table)
    c.store(x, y, ints([0, 4, 4, 4, 4]), ints([4, 4, 9, 35]))  # block 0's slots 0 to 3
    c.store(r.k, r.v, *r.at())
    for bad in (c._c.n_blocks, -1, -(1 << 31), (1 << 31) - 1):
        table[3, 2] = bad
        c.block_table.copy_(table)
        c.status.zero_()
        k, v = c.read(*r.at(), rows=5)
        assert c.status.tolist() == [0, 0, 0, 2]
        for got, own, zero in ((k, r.k, x), (v, r.v, y)):
            want = torch.cat([own[:2], zero[:3]])
            if kind == "packed":
                want = torch.from_numpy(ref.held(want.float().cpu().numpy(), r.name)[2]).to(r.dtype).cuda()
            assert bits(got.contiguous()).equal(bits(want.contiguous())), bad


@pytest.mark.parametrize("size,eps", [(1e25, 1e-6), (1e25, 0.0), (1e38, 1e-6), (1e19, 1e-3), (1e-19, 0.0), (1e-25, 0.0), (1e-25, 1e-12), (1e-38, 0.0),
                                      (1e-25, 1e-38), (1e-25, 1e-40), (1e-30, 1e-44), (1e-30, 1e10), (1e25, 1e38), (1e-15, 1e-30)])
@pytest.mark.parametrize("dim,heads", [(64, 5), (128, 3), (256, 2)])
def test_norms_of_large_and_small_heads(dim, heads, size, eps):
    """Heads whose squares are past the range of 32 bits, or below it, beside ordinary ones."""
    say("case norms", dim, size, eps)
    r = Rows(dim, [5, 1, 11], [3, 0, 20], dim=dim, q_heads=heads, kv_heads=2, norm="f32", rot=32, fused=False)
    for x in (r.q, r.k):
        x[::2, 1] = (x[::2, 1].float() * size).clamp(-3e38, 3e38).to(r.dtype)
        x[1::4, 0] = (x[1::4, 0].float() * size).clamp(-3e38, 3e38).to(r.dtype)
    r.kw["eps"] = float(np.float32(eps))  # what the call hands on
    assert np.isfinite(r.wants()[0]).all() and np.isfinite(r.wants()[1]).all()
    r.check_paged()
    r.check_packed()


@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_norms_of_heads_that_are_not_numbers(eps):
    """They come out as none, and those beside them as ever; so do heads of zeros without an eps."""
    say("case norms none", eps)
    r = Rows(3, [9], [0], dim=128, q_heads=3, kv_heads=2, norm="type", rot=0, fused=False)
    want = r.cache.store(r.k, r.v, *r.at(), q=r.q, eps=eps, **r.kw).clone()
    r.q[0, 0, 5], r.q[1, 1, 127], r.q[2, 2, 0] = float("nan"), float("inf"), float("-inf")
    r.q[3, 0] = 0
    got = r.cache.store(r.k, r.v, *r.at(), q=r.q, eps=eps, **r.kw)
    assert got[0, 0].isnan().all() and got[1, 1, 127].isnan() and got[2, 2, 0].isnan() and (got[3, 0].isnan().all() if eps == 0 else got[3, 0].eq(0).all())
    same = torch.ones(9, 3, dtype=torch.bool, device="cuda")
    for i, h in ((0, 0), (1, 1), (2, 2), (3, 0)):
        same[i, h] = False
    assert bits(got[same]).equal(bits(want[same]))


def test_rows_that_share_memory_are_refused():
    """What a read writes, and the queries that a store reads and writes elsewhere; tensors side by side are fine."""
    import paper_2605_24259_amd as rkc
    r = Rows(1, [4, 3], [4, 9], q_heads=2, kv_heads=2, norm=None, rot=0)
    at = r.at()
    for c in (r.cache, r.packed):
        c.store(r.k, r.v, *at)
        want = c.read(*at, rows=7)
        flat, t = torch.zeros(9000, dtype=r.dtype, device="cuda"), torch.zeros(8, 4, 128, dtype=r.dtype, device="cuda")
        for k, v in ((t[:7, :2], t[:7, :2]), (t[:7, :2], t[1:, :2]), (t[1:, 1:3], t[:7, 2:]), (flat[:7 * 256].view(7, 2, 128), flat[8: 8 + 7 * 256].view(7, 2, 128)),
                     (flat[:7 * 256].view(7, 2, 128), flat.as_strided((7, 2, 128), (512, 256, 1)))):
            with pytest.raises(rkc.RkcError, match="share"):
                c.read(*at, rows=7, k=k, v=v)
            assert flat.eq(0).all() and t.eq(0).all()
        pair, outer = (torch.zeros(n, dtype=r.dtype, device="cuda") for n in ((7, 2, 2, 128), (2, 2, 7, 128)))
        for k, v in ((t[:7, :2], t[:7, 2:]), (t[:7, 2:], t[:7, :2]), (t[:7, ::2], t[:7, 1::2]), (pair[:, :, 1], pair[:, :, 0]), (outer[0].transpose(0, 1), outer[1].transpose(0, 1)),
                     (outer[:, 0].transpose(0, 1), outer[:, 1].transpose(0, 1)), (flat[:1792].view(7, 2, 128), flat[1792: 3584].view(7, 2, 128))):
            got = c.read(*at, rows=7, k=k, v=v)
            assert got[0] is k and got[1] is v and all(bits(a.contiguous()).equal(bits(b)) for a, b in zip(got, want))
        q = torch.zeros(8, 4, 128, dtype=r.dtype, device="cuda")
        q[:7, :2] = r.q
        for out in (q[1:, :2], q[:7, 1:3]):
            with pytest.raises(rkc.RkcError, match="share"):
                c.store(r.k, r.v, *at, q=q[:7, :2], q_out=out)
        assert bits(c.store(r.k, r.v, *at, q=q[:7, :2], q_out=q[:7, 2:]).contiguous()).equal(bits(r.q.contiguous()))
        assert bits(c.store(r.k, r.v, *at, q=q[:7, :2], q_out=q[:7, :2]).contiguous()).equal(bits(r.q.contiguous()))


@pytest.mark.parametrize("kind", ["cache", "packed"])
def test_outputs_of_attention_that_share_memory_are_refused(kind):
    """Outputs in the queries' place are fine, beside them too, over other rows or heads of them not."""
    import paper_2605_24259_amd as rkc
    r = Rows(1, [4, 3], [4, 9], q_heads=2, kv_heads=2, norm=None, rot=0)
    c, at = getattr(r, kind), r.at()
    c.store(r.k, r.v, *at)
    x = torch.zeros(8, 4, 128, dtype=r.dtype, device="cuda")
    x[:7, :2] = r.q
    want = c.attend(x[:7, :2], *at, max_rows=4)[0]
    for out in (x[1:, :2], x[:7, 1:3]):
        with pytest.raises(rkc.RkcError, match="share"):
            c.attend(x[:7, :2], *at, max_rows=4, out=out)
    assert bits(c.attend(x[:7, :2], *at, max_rows=4, out=x[:7, 2:])[0].contiguous()).equal(bits(want))
    assert bits(c.attend(x[:7, :2], *at, max_rows=4, out=x[:7, :2])[0].contiguous()).equal(bits(want))
