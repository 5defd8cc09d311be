"""Attention over a cache of 4 bits in the forms that only large batches take: many sequences over the blocks of one pool, which
keeps the plain implementation small.  Tolerances as in test_gpu_cache.py."""
import numpy as np
import pytest
import torch  # (before the library, which takes the HIP runtime that is there)

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
    want = c.attend_at_once()
    out, lse = run(c)
    check_attend(c, out, lse, want=want)
    again = run(c)
    assert out.equal(again[0]) and lse.equal(again[1])
