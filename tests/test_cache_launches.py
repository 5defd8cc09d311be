"""Sizes past what the runtime launches are refused before anything is enqueued: on the CPU, where a launch would fail with
another status."""
import ctypes

import pytest

from tests.test_cache_abi import call, lib, structs  # noqa: F401

UNSUPPORTED, SCRATCH, NO_GPU = -4, -5, -6
BIG = dict(d_scratch=1 << 40, scratch_bytes=1 << 62)


def sized(seqs, heads, length, group=1, rows=1, **kw):
    c, a, e = structs()
    c.n_seqs, c.kv_heads, c.max_pages, c.page_tokens = seqs, heads, -(-length // 1024), 1024
    c.k_slot_stride = c.v_slot_stride = heads * 128
    c.k_block_stride = c.v_block_stride = 1024 * heads * 128
    a.n_rows, a.q_heads, a.max_rows, a.max_len = seqs * rows, heads * group, rows, length
    a.q_row_stride = a.out_row_stride = heads * group * 128
    e.max_len = length
    for x in (a, e):
        x.weight_seq_stride, x.weight_head_stride = heads * length, length
        x.d_scratch, x.scratch_bytes = BIG["d_scratch"], BIG["scratch_bytes"]
    for k, v in kw.items():
        setattr(a, k, v)
    return c, a, e


def on_cpu():
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are not real: for a machine without a GPU")


@pytest.mark.parametrize("name,size,kw", [
    ("rkc_attend", (1 << 20, 16, 2048), {}),                                             # its own lanes
    ("rkc_attend", (1 << 20, 1, 1 << 26), dict(d_weight=0x300000)),                      # the account's, from kept scores
    ("rkc_attend", (1024, 8, 1 << 20), dict(d_weight=0x300000, d_row_start=0x310000)),   # the account's, from the keys
    ("rkc_attend", (1024, 8, 1 << 20, 17, 1), dict(d_weight=0x300000, d_parent=0x310000)),
    ("rkc_weigh", (1024, 8, 1 << 20), dict(d_weight=0x300000)),
    ("rkc_weigh", (1 << 20, 1, 1 << 26), dict(d_weight=0x300000)),
    ("rkc_evict", (1024, 8, 1 << 20), {}),
    ("rkc_evict", (1 << 20, 1, 1 << 20), {})])
def test_too_many_lanes(lib, name, size, kw):  # noqa: F811
    on_cpu()
    c, a, e = sized(*size, **kw)
    assert call(lib, name, c, e if name == "rkc_evict" else a) == UNSUPPORTED


@pytest.mark.parametrize("name,size,kw", [
    ("rkc_attend", (1 << 20, 1, 2048), {}), ("rkc_attend", (1024, 8, 1 << 17), dict(d_weight=0x300000)), ("rkc_weigh", (1024, 8, 1 << 17), dict(d_weight=0x300000)),
    ("rkc_attend", (1024, 8, 1 << 17), dict(d_weight=0x300000, d_row_start=0x310000)), ("rkc_evict", (1024, 8, 1 << 17), {})])
def test_fewer_are_launched(lib, name, size, kw):  # noqa: F811
    on_cpu()
    c, a, e = sized(*size, **kw)
    assert call(lib, name, c, e if name == "rkc_evict" else a) == NO_GPU


def test_the_size_is_told_before_the_scratch(lib):  # noqa: F811
    c, a, e = sized(1024, 8, 1 << 20, d_weight=0x300000, d_row_start=0x310000)
    a.d_scratch = 0
    assert call(lib, "rkc_attend", c, a) == UNSUPPORTED
    assert lib.rkc_attend_scratch_bytes(ctypes.byref(c), ctypes.byref(a)) >= 0


def test_an_account_wants_the_queries_left_alone(lib):  # noqa: F811
    c, a, e = structs()
    a.d_weight, a.d_out = 0x300000, a.d_q
    assert call(lib, "rkc_attend", c, a) == -3
