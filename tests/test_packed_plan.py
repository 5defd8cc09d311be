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
