"""Rows of a paged cache and the cache of 4 bits on the CPU: exports and layouts of include/rkc_packed.h, the host-side
checks, which return before any HIP call, and the plain implementation itself."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

from tests import packed_reference as ref
from tests.test_cache_abi import lib, structs  # noqa: F401
from tests.test_cache_launches import on_cpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "rkc_packed.h")


def test_exports_every_declared_function(lib):  # noqa: F811
    import paper_2605_24259_amd as rkc
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    decl = set(re.findall(r"\b(rkc_[a-z_]+)\s*\(", text))
    assert decl == set(rkc.packed.PACKED_EXPORTS)
    out = subprocess.check_output(["nm", "-D", "--defined-only", rkc.LIB_PATH], text=True)
    assert decl <= set(re.findall(r"\bT (rkc_\w+)", out))


def test_layouts_match_header(tmp_path):
    from paper_2605_24259_amd import packed, rows
    structs_ = {"rkc_packed": packed._Packed, "rkc_rows": rows._Rows}
    lines = [f'printf("%zu %zu\\n", sizeof({s}), offsetof({s}, {f}));' for s, t in structs_.items() for f, _ in t._fields_]
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include "rkc_packed.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "t")])
    got = [tuple(map(int, x.split())) for x in subprocess.check_output([str(tmp_path / "t")], text=True).splitlines()]
    assert got == [(ctypes.sizeof(t), getattr(t, f).offset) for t in structs_.values() for f, _ in t._fields_]
    assert re.search(rf"\bRKC_MAX_AXES {rows.MAX_AXES}\b", open(HEADER).read())


def fine():
    """A cache, the same in 4 bits, rows and an attention that are fine; the addresses are aligned and never used."""
    from paper_2605_24259_amd import packed, rows
    c, a, _ = structs()
    p, r = packed._Packed(), rows._Rows()
    p.n_seqs, p.n_blocks, p.max_pages, p.page_tokens, p.kv_heads, p.head_dim = 4, 300, 64, 16, 2, 128
    p.head_stride = 16 * 136
    p.block_stride = 2 * p.head_stride
    p.d_pool, p.d_block_table, p.d_status = 0x10000, 0x30000, 0x40000
    r.n_rows, r.q_heads, r.max_len, r.n_freq, r.axes, r.eps = 4, 8, 1024, 64, 3, 1e-6
    r.k_row_stride = r.v_row_stride = 256
    r.k_head_stride = r.v_head_stride = r.q_head_stride = r.q_out_head_stride = 128
    r.q_row_stride = r.q_out_row_stride = 1024
    r.d_k, r.d_v, r.d_q, r.d_q_out, r.d_row_offset, r.d_length = range(0x100000, 0x160000, 0x10000)
    r.d_position, r.d_axis, r.d_freq, r.d_q_norm, r.d_k_norm = range(0x160000, 0x1b0000, 0x10000)
    return c, p, r, a


def call(lib, name, c, x):  # noqa: F811
    return getattr(lib, name)(ctypes.byref(c), ctypes.byref(x), None)


@pytest.mark.parametrize("fault,status", [
    (dict(d_pool=0), -1), (dict(d_block_table=0), -1), (dict(d_pool=0x10008), -2), (dict(d_status=0x40002), -2), (dict(n_seqs=-1), -3),
    (dict(n_blocks=0), -3), (dict(max_pages=0), -3), (dict(kv_heads=0), -3), (dict(reserved=1), -3), (dict(block_stride=-16), -3),
    (dict(block_stride=8), -3), (dict(block_stride=1 << 32), -3), (dict(head_stride=24), -3), (dict(head_stride=1 << 41), -3),
    (dict(dtype=2), -4), (dict(head_dim=96), -4), (dict(page_tokens=8), -4), (dict(page_tokens=48), -4), (dict(page_tokens=2048), -4)])
def test_packed_cache_checks(lib, fault, status):  # noqa: F811
    _, p, r, a = fine()
    for k, v in fault.items():
        setattr(p, k, v)
    for name, x in (("rkc_packed_store", r), ("rkc_packed_read", r), ("rkc_packed_attend", a)):
        assert call(lib, name, p, x) == status, name


BOTH = [(dict(d_k=0), -1), (dict(d_v=0), -1), (dict(d_row_offset=0), -1), (dict(d_length=0), -1), (dict(d_k=0x100008), -2),
        (dict(d_v=0x110004), -2), (dict(d_row_offset=0x140002), -2), (dict(n_rows=-1), -3), (dict(max_len=-1), -3), (dict(max_len=1025), -3),
        (dict(k_row_stride=-8), -3), (dict(v_head_stride=12), -3), (dict(k_row_stride=1 << 41), -3)]
STORE = [(dict(d_q_out=0), -1), (dict(d_freq=0), -1), (dict(d_q=0x120008), -2), (dict(d_q_out=0x130002), -2), (dict(d_position=0x160001), -2),
         (dict(d_axis=0x170002), -2), (dict(d_freq=0x180001), -2), (dict(d_q_norm=0x190001), -2), (dict(d_k_norm=0x1a0002, norm_f32=1), -2),
         (dict(q_heads=-1), -3), (dict(q_heads=1 << 17), -3), (dict(n_freq=-8), -3), (dict(n_freq=12), -3), (dict(n_freq=72), -3),
         (dict(interleaved=2), -3), (dict(norm_f32=-1), -3), (dict(eps=-1.0), -3), (dict(eps=float("nan")), -3), (dict(eps=float("inf")), -3),
         (dict(axes=0), -3), (dict(axes=9), -3), (dict(d_axis=0), -3), (dict(d_position=0), -3), (dict(q_row_stride=4), -3),
         (dict(q_out_row_stride=512), -3), (dict(q_out_head_stride=0), -3), (dict(d_q_out=0x120000, q_row_stride=2048), -3)]
READ = [(dict(k_row_stride=128), -3), (dict(k_head_stride=0), -3), (dict(v_row_stride=0), -3), (dict(v_head_stride=120), -3)]


@pytest.mark.parametrize("fault,status,names", [(f, s, ("store", "read")) for f, s in BOTH] + [(f, s, ("store",)) for f, s in STORE]
                         + [(f, s, ("read",)) for f, s in READ])
def test_rows_checks(lib, fault, status, names):  # noqa: F811
    c, p, r, _ = fine()
    for k, v in fault.items():
        setattr(r, k, v)
    for n in names:
        assert call(lib, "rkc_" + n, c, r) == status, n
        assert call(lib, "rkc_packed_" + n, p, r) == status, n


def test_slots_keep_apart(lib):  # noqa: F811
    """Slots that share memory are refused where they are written."""
    for field, value in (("k_head_stride", 0), ("v_slot_stride", 128), ("k_block_stride", 8)):
        c, p, r, _ = fine()
        setattr(c, field, value)
        assert call(lib, "rkc_store", c, r) == -3, field
    for field, value in (("head_stride", 16 * 135), ("head_stride", 0), ("block_stride", 16 * 136)):
        c, p, r, _ = fine()
        setattr(p, field, value)
        assert call(lib, "rkc_packed_store", p, r) == -3, field


def test_null_and_nothing_to_do(lib):  # noqa: F811
    c, p, r, a = fine()
    for x, names, y in ((c, ("rkc_store", "rkc_read"), r), (p, ("rkc_packed_store", "rkc_packed_read"), r), (p, ("rkc_packed_attend",), a)):
        for n in names:
            assert getattr(lib, n)(None, ctypes.byref(y), None) == -1
            assert getattr(lib, n)(ctypes.byref(x), None, None) == -1
    r.n_rows = a.n_rows = 0
    for x, names, y in ((c, ("rkc_store", "rkc_read"), r), (p, ("rkc_packed_store", "rkc_packed_read"), r), (p, ("rkc_packed_attend",), a)):
        for n in names:
            assert call(lib, n, x, y) == 0
    c, p, r, a = fine()
    c.n_seqs = p.n_seqs = 0
    p.d_pool = p.d_block_table = c.d_k = c.d_v = c.d_block_table = r.d_k = a.d_q = 0
    for x, names, y in ((c, ("rkc_store", "rkc_read"), r), (p, ("rkc_packed_store", "rkc_packed_read"), r), (p, ("rkc_packed_attend",), a)):
        for n in names:
            assert call(lib, n, x, y) == 0


@pytest.mark.parametrize("fault,status", [
    (dict(d_q=0), -1), (dict(d_out=0), -1), (dict(d_lse=0), -1), (dict(d_q=0x50004), -2), (dict(max_len=1025), -3), (dict(q_heads=3), -3),
    (dict(softcap=-1.0), -3), (dict(scale=float("nan")), -3), (dict(out_row_stride=512), -3), (dict(d_parent=0x200000, max_rows=257), -4),
    (dict(d_weight=0x300000), -4), (dict(d_weight_in=0x300000), -4)])
def test_attention_checks(lib, fault, status):  # noqa: F811
    _, p, _, a = fine()
    for k, v in fault.items():
        setattr(a, k, v)
    assert call(lib, "rkc_packed_attend", p, a) == status


def test_scratch(lib):  # noqa: F811
    _, p, _, a = fine()
    p.max_pages, a.max_len = 1024, 16384
    need = lib.rkc_packed_attend_scratch_bytes(ctypes.byref(p), ctypes.byref(a))
    assert need > 0 and call(lib, "rkc_packed_attend", p, a) == -5
    a.scratch_bytes, a.d_scratch = need, 0x100080
    assert call(lib, "rkc_packed_attend", p, a) == -2
    a.scratch_bytes, a.d_scratch = need - 1, 0x100000
    assert call(lib, "rkc_packed_attend", p, a) == -5
    assert lib.rkc_packed_attend_scratch_bytes(None, ctypes.byref(a)) == 0
    for rows, length in ((1, 1 << 20), (64, 1 << 20), (4000, 1 << 16)):
        p.max_pages, a.max_rows, a.max_len = length // 16, rows, length
        assert lib.rkc_packed_attend_scratch_bytes(ctypes.byref(p), ctypes.byref(a)) <= 256 * 4 * (1 << 20)


def test_too_many_lanes(lib):  # noqa: F811
    """Sizes past what the runtime launches are refused, and smaller ones are not (without a GPU: its error)."""
    on_cpu()
    _, p, _, a = fine()
    p.n_seqs, p.kv_heads, p.max_pages, p.page_tokens, p.head_stride = 1 << 20, 16, 2, 1024, 1024 * 136
    p.block_stride = 16 * p.head_stride
    a.n_rows, a.q_heads, a.max_rows, a.max_len = 1 << 20, 16, 1, 2048
    a.q_row_stride = a.out_row_stride = 16 * 128
    a.d_scratch, a.scratch_bytes = 1 << 40, 1 << 62
    assert call(lib, "rkc_packed_attend", p, a) == -4
    p.kv_heads = a.q_heads = 1
    assert call(lib, "rkc_packed_attend", p, a) == -6


@pytest.mark.parametrize("rows,status", [(0x7fffffff, -4), (0x7ffffff0, -4), (1 << 20, -6)])
def test_too_many_rows(lib, rows, status):  # noqa: F811
    """A workgroup of 256 lanes has 64 rows at most: 2^31 rows are 2^33 lanes, past the 2^32 of a launch, whatever is added to
    the rows on the way to their workgroups; 2^20 rows are not (without a GPU: its error)."""
    on_cpu()
    c, p, r, _ = fine()
    r.n_rows, r.q_heads, r.d_position, r.d_axis = rows, 1, 0, 0
    for heads in (1, 2):
        c.kv_heads = p.kv_heads = heads
        for name, x in (("rkc_store", c), ("rkc_read", c), ("rkc_packed_store", p), ("rkc_packed_read", p)):
            assert call(lib, name, x, r) == status, (name, heads)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_the_reference_holds_the_nearest(dtype):
    """Of the sixteen values, times the least scale that reaches the largest."""
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.standard_normal((40, 32)), rng.standard_normal((40, 32)) * 2.0 ** rng.integers(-20, 9, (40, 1)),
                        np.repeat([[7.0], [7.0 + 2.0 ** -20], [3.5], [0.0]], 32, 1)]).astype(np.float32)
    code, scale, value = ref.held(x, dtype)
    every = np.concatenate([ref.VALUES, -ref.VALUES])
    for row, s, v in zip(x.astype(np.float64), scale[:, 0].astype(int), value):
        by = 2.0 ** (s - 127)
        assert np.abs(row).max() <= 7 * by and (np.abs(row).max() > 3.5 * by or s == 1)
        near = np.abs(row[:, None] / by - every).min(1)
        assert np.array_equal(np.abs(row / by - v / by), near)
    for half, to in ((0.25, 0), (0.75, 1), (1.25, 1), (1.75, 2), (2.5, 2), (3.5, 4), (5, 4)):
        y = np.full((1, 32), half, np.float32)
        y[0, 0] = 6
        assert ref.held(y, dtype)[2][0, 1] == to
    kc = ref.joined(*[np.zeros((2, 3, 16, 64), np.uint8)] * 2, *[np.zeros((2, 3, 16, 2), np.uint8)] * 2)
    assert kc.shape == (2, 3, 16 * 68)
    assert np.array_equal(ref.values(code, scale), value)


def test_angles_of_the_reference():
    for p, f in ((12345, 0.7), (-7, 1.0), (1 << 30, float(np.float32(0.1)))):
        t = ref.whole_angle(p, f)
        assert abs(t) <= 3.1416 and abs(np.cos(t) - np.cos(p * f)) < 1e-6
