"""The operators on a paged KV cache where tables, masks and values are at an edge; the tolerances are those of
test_gpu_cache.py."""
import numpy as np
import pytest

from tests import cache_reference as ref
from tests.gpu_util import say
from tests.test_gpu_cache import UNIT, bush, check_attend, check_weigh, gpu_cache, ints, mask, run_attend

pytestmark = pytest.mark.gpu

NEVER = 1 << 30


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,kv_heads,group,lens,rows,seeing", [
    (64, 1, 1, [320, 192], 192, 128), (64, 2, 4, [64, 64], 64, 32), (128, 1, 1, [500, 256], 256, 128), (256, 1, 1, [512, 160], 160, 128),
    (128, 8, 4, [1024] * 4, 256, 64)])
def test_row_tiles_of_padding_alone(dtype, dim, kv_heads, group, lens, rows, seeing):
    """Rows that see nothing fill whole row tiles, in tables that end with the last sequence's last page."""
    say("case padding", dtype, dim, kv_heads, group, lens, rows)
    start = [max(0, n - rows + i - 40) if i < seeing else NEVER for n in lens for i in range(rows)]
    c = ref.Case(dim, lens, [rows] * len(lens), kv_heads=kv_heads, group=group, dim=dim, dtype=dtype, row_start=start)
    c.table = c.table[:, : -(-max(lens) // c.page)].contiguous()  # no spare page
    out, lse = run_attend(c)
    check_attend(c, out, lse)
    seen = np.tile(np.arange(rows) < seeing, len(lens))
    assert np.isneginf(lse.cpu().numpy()[~seen]).all() and (out.cpu()[~seen] == 0).all() and lse.cpu()[seen].isfinite().all()


@pytest.mark.parametrize("prefix", [False, True])
@pytest.mark.parametrize("late", [1, "rows", NEVER])
@pytest.mark.parametrize("dim,group,rows", [(64, 2, 3), (128, 4, 4), (256, 1, 9), (64, 1, 40), (64, 2, 70), (128, 3, 90), (256, 2, 70)])
def test_trees_that_start_past_their_base(prefix, late, dim, group, rows):
    """A tree's rows see their own slot and their ancestors' wherever row_start lies: past the base it takes the history away
    and nothing else.  For all rows of one sequence, for the first 32 packed rows of another, which fill a wave, and
    in long sequences that are cut."""
    say("case late trees", prefix, late, dim, group, rows)
    long = 1600 if rows * group <= 16 else 700
    lens, ns, start, first = [rows + 20, rows + 75, rows + long, rows], [rows] * 4, [], max(1, 32 // group)
    for s, n in enumerate(lens):
        base = n - rows
        past = base + 1 if late == 1 else base + rows if late == "rows" else NEVER
        start += [past if s != 1 or i < first else 10 for i in range(rows)]
    c = ref.Case(rows + dim, lens, ns, kv_heads=2, group=group, dim=dim, dtype="float16" if prefix else "bfloat16", parent=sum((bush(rows, s) for s in range(4)), []),
                 row_start=start, prefix=[7, 40, 100, 0] if prefix else None, bias=dim == 128)
    want = c.attend()
    assert np.isfinite(want[1]).all()
    out, lse = run_attend(c)
    check_attend(c, out, lse, want)
    g, w = gpu_cache(c), c.weight.cuda()
    q, o, n = c.q.cuda(), ints(c.offset), ints(c.lens)
    check_weigh(c, g.weigh(q, lse, o, n, weight=w, decay=0.5, **mask(c, max_len=max(lens))), lse, 0.5, c.weight)
    out, lse, got = g.attend(q, o, n, weight=w, decay=0.5, **mask(c, max_len=max(lens)))
    check_attend(c, out, lse, want)
    check_weigh(c, got, lse, 0.5, c.weight)
    assert not g.status.any().item()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("dim,group,rows,lens", [(64, 3, 1, [200, 1700]), (128, 4, 1, [131, 2000]), (256, 2, 1, [200, 700]),
                                                 (128, 2, 6, [200, 1800]), (64, 2, 40, [300, 900]), (128, 1, 150, [400, 700])])
def test_infinities_that_all_rows_see(dtype, dim, group, rows, lens):
    """Infinite values, and NaN, at slots of tiles that every row sees whole: infinite outputs, of the value's sign, NaN where
    both signs meet or a NaN is, and all other elements as always.  Each column has a slot of its own, so that what a
    weight loses to rounding takes both signs and zero."""
    say("case infinities", dtype, dim, group, rows, lens)
    plain = ref.Case(dim + rows, lens, [rows] * 2, kv_heads=1, group=group, dim=dim, dtype=dtype, parent=bush(rows) * 2)
    base, free = run_attend(plain)
    c = ref.Case(dim + rows, lens, [rows] * 2, kv_heads=1, group=group, dim=dim, dtype=dtype, parent=bush(rows) * 2)

    def put(s, slot, col, value):
        c.v[c.table[s, slot // c.page], slot % c.page, :, col] = value
    for s, n in enumerate(lens):
        history = (n - rows) // 64 * 64
        for col in range(0, dim, 2):
            put(s, (col * 7 + 3 * s) % history, col, float("inf" if col % 4 else "-inf"))
        put(s, 5, 8, float("inf"))  # beside a negative one
        put(s, 9, 12, float("nan"))
    o, z = c.attend()
    out, lse = run_attend(c)
    got = out.double().cpu().numpy()
    assert np.isinf(o).sum() >= o.size // 2 - 3 * o.size // dim and np.isnan(o[..., 12]).all() and np.isnan(o[..., 8]).all()
    check_attend(c, out, lse, (o, z))
    import torch
    assert torch.equal(out[..., 1::2], base[..., 1::2]) and torch.equal(lse, free)


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dim,group,rows", [(64, 1, 3), (64, 1, 40), (128, 4, 60), (256, 2, 30), (128, 4, 100)])
def test_parents_are_flagged_where_sequences_are_cut(dim, group, rows, bias):
    """A parent that is none is taken for -1 and told of by each call, wherever in its sequence the tree lies."""
    import torch

    import paper_2605_24259_amd as rkc
    say("case parents", dim, group, rows, bias)
    lens = [2000, 1990, 40 + rows, 1700]
    c = ref.Case(dim + rows, lens, [rows] * 4, kv_heads=1, group=group, dim=dim, parent=bush(rows) * 4, bias=bias)
    g, told = gpu_cache(c), rkc.cache.CS_PARENT
    q, o, n, m = c.q.cuda(), ints(c.offset), ints(c.lens), mask(c, max_len=2000)
    wrong = m["parent"].clone()
    wrong[rows - 1], wrong[rows + 1], wrong[2 * rows + 2] = rows - 1, -2, 1 << 30
    right = wrong.clone()
    for at in (rows - 1, rows + 1, 2 * rows + 2):
        right[at] = -1
    want = g.attend(q, o, n, **dict(m, parent=right))
    account = g.weigh(q, want[1], o, n, **dict(m, parent=right))
    assert not g.status.any().item()
    got = g.attend(q, o, n, **dict(m, parent=wrong))
    assert g.status.tolist() == [told, told, told, 0]
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    g.status.zero_()
    assert torch.equal(g.weigh(q, want[1], o, n, **dict(m, parent=wrong)), account)
    assert g.status.tolist() == [told, told, told, 0]


@pytest.mark.parametrize("account", [False, True])
def test_rows_where_none_may_be(account):
    """max_rows of 0 and rows all the same: their sequences are left out and told of, like any that have too many."""
    import torch

    import paper_2605_24259_amd as rkc
    say("case no rows allowed", account)
    c = ref.Case(3, [50, 2000, 7], [2, 0, 1])
    g, w = gpu_cache(c), c.weight.cuda()
    out, to = torch.full_like(c.q, 5.0).cuda(), torch.full_like(w, 3.0)
    more = dict(weight=w, weight_out=to, decay=0.5) if account else {}
    g.attend(c.q.cuda(), ints(c.offset), ints(c.lens), out=out, **mask(c, max_rows=0, max_len=2000), **more)
    assert g.status.tolist() == [rkc.cache.CS_LENGTH, 0, rkc.cache.CS_LENGTH] and (out == 5).all()
    assert (to[0] == 3).all() and (to[2] == 3).all() and torch.equal(to[1, :, :2000], w[1, :, :2000] * 0.5 if account else torch.full_like(to[1, :, :2000], 3.0))


@pytest.mark.parametrize("softcap", [1e3, 1e6])
@pytest.mark.parametrize("dim,group,rows,n", [(64, 2, 5, 90), (128, 4, 4, 2000), (256, 2, 6, 300), (64, 2, 40, 300), (128, 3, 60, 700), (256, 2, 70, 300)])
@pytest.mark.parametrize("what", ["row", "slot"])
def test_far_caps_beside_large_scores(softcap, dim, group, rows, n, what):
    """A row's scores are capped as exactly beside a row, or a slot that it does not see, whose scores reach the cap as
    they are without: to 2^-20 (8 + the largest |scale| |q| |k| of the slots that the row itself sees)."""
    import torch
    say("case caps", softcap, dim, group, rows, n, what)
    c = ref.Case(dim + rows, [n], [rows], kv_heads=1, group=group, dim=dim, softcap=softcap, parent=bush(rows))
    base, big = n - rows, softcap / 4
    if what == "row":
        c.q[1] *= big
    else:
        c.k[c.table[0, (base + 1) // 16], (base + 1) % 16] *= big
    see = c.seen(0)[0]
    k = np.linalg.norm(c.slots(c.k, 0, 0), axis=-1)
    q = np.linalg.norm(c.q.double().numpy(), axis=-1)
    top = np.where(see, k[None], 0).max(1)
    a = 2.0 ** -20 * (8 + c.scale * q * top[:, None])
    assert a.max() > 20 * a.min()  # scores that reach the cap are there, and such that do not
    o, z = c.attend()
    out, lse = run_attend(c)
    assert np.all(np.abs(lse.double().cpu().numpy() - z) <= a), (np.abs(lse.double().cpu().numpy() - z) / a).max()
    vmax = np.nan_to_num(c.v.double().numpy(), nan=0, posinf=0, neginf=0).__abs__().max()
    u = UNIT["bfloat16"]
    assert np.all(np.abs(out.double().cpu().numpy() - o) <= u * (vmax + np.abs(o)) + a[..., None] * vmax)
    # each row's own part of the account, of a call with this row's sum alone
    quiet = int(np.argmin(a.max(1)))
    only = torch.full(z.shape, -np.inf, dtype=torch.float32)
    only[quiet] = torch.from_numpy(z[quiet]).float()
    w = gpu_cache(c).weigh(c.q.cuda(), only.cuda(), ints(c.offset), ints(c.lens), **mask(c)).double().cpu().numpy()[0, 0, :n]
    want = c.weigh(only.double().numpy(), 1.0)[0, 0]
    assert np.all(np.abs(w - want) <= (a[quiet].max() + 2.0 ** -23 * np.abs(z[quiet]).max() + 2.0 ** -22) * want + 1e-30)


@pytest.mark.parametrize("dim,group,rows,lens", [(64, 2, 1, [300, 40]), (128, 4, 3, [2500, 90]), (256, 1, 4, [900, 30]), (64, 1, 200, [900, 200]), (128, 4, 40, [700, 90])])
def test_outputs_in_place_of_queries(dim, group, rows, lens):
    """Outputs may go where the queries were, but not with an account, for which the queries may be read again."""
    import torch

    import paper_2605_24259_amd as rkc
    say("case in place", dim, group, rows, lens)
    c = ref.Case(dim + rows, lens, [rows] * 2, group=group, dim=dim)
    want = run_attend(c)
    g, q, m = gpu_cache(c), c.q.cuda(), mask(c, max_len=max(lens))
    o, n, w = ints(c.offset), ints(c.lens), c.weight.cuda()
    for kw in (dict(weight=w), dict(weight_out=w)):
        with pytest.raises(rkc.RkcError) as e:
            g.attend(q, o, n, out=q, **kw, **m)
        assert e.value.status == -3 and torch.equal(q, c.q.cuda()) and torch.equal(w, c.weight.cuda())
    out, lse = g.attend(q, o, n, out=q, **mask(c))
    assert out is q and torch.equal(out, want[0]) and torch.equal(lse, want[1])
