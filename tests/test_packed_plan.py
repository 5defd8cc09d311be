"""Which kernel the attention over 4 bits takes and how it cuts sequences, on the CPU."""
import ctypes

import pytest

from tests.test_cache_abi import lib, structs  # noqa: F401


class Plan(ctypes.Structure):
    """rkc_plan (rkc_cache_dev.h)."""
    _fields_ = [("few", ctypes.c_bool)] + [(n, ctypes.c_int) for n in ("units", "tiles", "rows", "waves", "chunk", "splits")] + \
        [("sorted", ctypes.c_bool)] + [(n, ctypes.c_size_t) for n in ("part_at", "stat_at", "bytes")] + \
        [("keep", ctypes.c_bool), ("wide", ctypes.c_int), ("score_at", ctypes.c_size_t)]


def plan_of(lib, seqs, heads, dim, group, rows, max_len, tree=False):  # noqa: F811
    f = lib._Z15rkc_packed_planPK9rkc_cachePK13rkc_attention
    c, a, _ = structs()
    f.argtypes, f.restype = [ctypes.POINTER(type(c)), ctypes.POINTER(type(a))], Plan
    c.n_seqs, c.kv_heads, c.head_dim, c.max_pages = seqs, heads, dim, -(-max_len // 16)
    a.q_heads, a.max_rows, a.max_len, a.n_rows = heads * group, rows, max_len, seqs * rows
    a.d_parent = 0x200000 if tree else 0
    p = f(ctypes.byref(c), ctypes.byref(a))
    assert p.units == seqs * heads * p.tiles and p.splits == max(1, -(-max_len // p.chunk))  # the fields are where they are taken to be
    return p


def whole(lib, seqs, heads, dim, max_len):  # noqa: F811
    p = plan_of(lib, seqs, heads, dim, 4, 1, max_len)
    assert p.few and p.rows == 16 and (p.waves == 4 or p.splits == 1)
    return p.waves == 8


@pytest.mark.parametrize("dim", [64, 128])
def test_whole_sequences_go_by_how_full_rounds_are(lib, dim):  # noqa: F811
    """Single tokens.  512 workgroups are on the card at once: sequences past 1,536 slots stay whole in a round that is full to
    three quarters, or in several, whatever makes up the units."""
    for seqs, heads in ((48, 8), (60, 8), (63, 8), (64, 8), (24, 16), (32, 16), (400, 1), (512, 1), (250, 2), (160, 8), (192, 8), (100, 16), (3000, 1)):
        assert all(whole(lib, seqs, heads, dim, n) for n in (100, 1536, 1537, 4096, 8000, 8192)), (seqs, heads)
        assert not whole(lib, seqs, heads, dim, 8193)
    # the next round is all but empty: up to 4,096 slots, where it does not last
    for seqs, heads in ((65, 8), (513, 1), (33, 16), (80, 8), (96, 8), (159, 8)):
        assert all(whole(lib, seqs, heads, dim, n) for n in (1536, 1537, 4096)), (seqs, heads)
        assert not whole(lib, seqs, heads, dim, 4097) and not whole(lib, seqs, heads, dim, 8192)
    for seqs, heads in ((1, 1), (4, 2), (32, 8), (47, 8), (383, 1)):
        assert whole(lib, seqs, heads, dim, 1536) and not whole(lib, seqs, heads, dim, 1537), (seqs, heads)


def test_wide_heads_are_never_whole_by_eight_waves(lib):  # noqa: F811
    assert not any(whole(lib, seqs, 8, 256, n) for seqs in (1, 64, 160) for n in (100, 1536, 8192))



# sequences, heads, elements of a head, packed rows (in groups of 4), slots, and whether the kernel of few rows was the faster, by a tenth or more
BETWEEN = [
    (4, 8, 64, 32, 500, True), (4, 8, 64, 96, 500, True), (64, 8, 64, 48, 1000, False), (64, 8, 64, 96, 1000, False), (16, 8, 64, 96, 4096, False),
    (1, 8, 64, 20, 32768, True), (1, 8, 64, 96, 32768, False), (8, 8, 64, 32, 32768, True), (8, 8, 64, 96, 32768, False), (64, 8, 64, 32, 4096, True),
    (64, 8, 64, 96, 4096, False), (40, 8, 64, 32, 8192, True), (40, 8, 64, 64, 8192, True),
    (4, 8, 128, 20, 500, True), (4, 8, 128, 96, 500, True), (64, 8, 128, 48, 1000, False), (64, 8, 128, 96, 1000, False), (16, 8, 128, 20, 4096, True),
    (16, 8, 128, 64, 4096, False), (1, 8, 128, 32, 32768, True), (1, 8, 128, 96, 32768, False), (8, 8, 128, 32, 32768, True), (8, 8, 128, 96, 32768, False),
    (64, 8, 128, 32, 4096, True), (64, 8, 128, 64, 4096, False), (64, 8, 128, 96, 4096, False), (40, 8, 128, 32, 8192, True), (40, 8, 128, 64, 8192, True),
    (4, 4, 256, 48, 500, True), (4, 4, 256, 96, 500, True), (64, 4, 256, 48, 1000, False), (64, 4, 256, 96, 1000, False), (16, 4, 256, 64, 4096, False),
    (1, 4, 256, 32, 32768, False), (1, 4, 256, 96, 32768, False), (8, 4, 256, 32, 32768, True), (8, 4, 256, 64, 32768, True), (8, 4, 256, 96, 32768, False),
    (64, 4, 256, 32, 4096, True), (64, 4, 256, 64, 4096, True), (64, 4, 256, 96, 4096, False), (16, 4, 256, 32, 8192, True),
    (40, 8, 128, 96, 8192, True), (16, 4, 256, 64, 8192, True)]


@pytest.mark.parametrize("seqs,heads,dim,packed,slots,few", BETWEEN)
def test_the_faster_kernel_is_taken(lib, seqs, heads, dim, packed, slots, few):  # noqa: F811
    """17 to 96 packed rows, where either kernel may be the faster."""
    p = plan_of(lib, seqs, heads, dim, 4, packed // 4, slots, tree=True)
    assert bool(p.few) == few and p.rows == (32 if few else 128) and p.tiles == -(-packed // p.rows)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("seqs,slots", [(1, 1), (4, 500), (64, 1000), (64, 8192), (1, 1 << 20)])
def test_packed_rows_of_either_kernel(lib, dim, seqs, slots):  # noqa: F811
    """Up to 16 by the one; more than 96, and trees of more than 32 rows, by the other."""
    for rows, group in ((1, 1), (1, 16), (16, 1), (4, 4)):
        p = plan_of(lib, seqs, 8, dim, group, rows, slots, tree=True)
        assert p.few and p.rows == 16 and p.tiles == 1
    for rows, group, tree in ((97, 1, False), (1, 97, False), (300, 1, False), (33, 1, True), (48, 2, True), (256, 4, True)):
        p = plan_of(lib, seqs, 8, dim, group, rows, slots, tree)
        assert not p.few and p.rows in (128, 256) and p.tiles == -(-rows * group // p.rows)
