"""The operators on a paged KV cache on the CPU: exports and layouts of include/rkc_cache.h, and the host-side checks,
which return before any HIP call."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "rkc_cache.h")


@pytest.fixture(scope="module")
def lib():
    import paper_2605_24259_amd as rkc
    if not os.path.exists(rkc.LIB_PATH):
        from paper_2605_24259_amd import build
        build.build()
    return rkc.load()


def test_exports_every_declared_function(lib):
    import paper_2605_24259_amd as rkc
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    decl = set(re.findall(r"\b(rkc_[a-z_]+)\s*\(", text))
    assert decl == set(rkc.cache.CACHE_EXPORTS)
    out = subprocess.check_output(["nm", "-D", "--defined-only", rkc.LIB_PATH], text=True)
    assert decl <= set(re.findall(r"\bT (rkc_\w+)", out))


def test_layouts_match_header(tmp_path):
    from paper_2605_24259_amd import cache
    structs = {"rkc_cache": cache._Cache, "rkc_attention": cache._Attention, "rkc_eviction": cache._Eviction}
    lines = [f'printf("%zu %zu\\n", sizeof({s}), offsetof({s}, {f}));' for s, t in structs.items() for f, _ in t._fields_]
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include "rkc_cache.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "t")])
    got = [tuple(map(int, x.split())) for x in subprocess.check_output([str(tmp_path / "t")], text=True).splitlines()]
    want = [(ctypes.sizeof(t), getattr(t, f).offset) for t in structs.values() for f, _ in t._fields_]
    assert got == want
    text = open(HEADER).read()
    for name, value in (("RKC_MAX_TREE_ROWS", cache.MAX_TREE_ROWS), ("RKC_CS_LENGTH", cache.CS_LENGTH),
                        ("RKC_CS_BLOCK", cache.CS_BLOCK), ("RKC_CS_PARENT", cache.CS_PARENT)):
        assert re.search(rf"\b{name}\b\s*=?\s*{value}\b", text)


def structs():
    """A cache of 4 sequences of up to 64 pages, an attention and an eviction that are fine but for their scratch; the
    addresses are aligned and never used."""
    from paper_2605_24259_amd import cache
    c, a, e = cache._Cache(), cache._Attention(), cache._Eviction()
    c.n_seqs, c.n_blocks, c.max_pages, c.page_tokens, c.kv_heads, c.head_dim = 4, 300, 64, 16, 2, 128
    c.k_block_stride = c.v_block_stride = 16 * 2 * 128
    c.k_slot_stride = c.v_slot_stride = 2 * 128
    c.k_head_stride = c.v_head_stride = 128
    c.d_k, c.d_v, c.d_block_table, c.d_status = 0x10000, 0x20000, 0x30000, 0x40000
    a.n_rows, a.q_heads, a.max_rows, a.max_len, a.scale = 4, 8, 1, 1024, 0.1
    a.q_row_stride = a.out_row_stride = 1024
    a.q_head_stride = a.out_head_stride = 128
    a.weight_seq_stride, a.weight_head_stride = 2048, 1024
    a.d_q, a.d_row_offset, a.d_length, a.d_out, a.d_lse = 0x50000, 0x60000, 0x70000, 0x80000, 0x90000
    e.max_len, e.weight_seq_stride, e.weight_head_stride = 1024, 2048, 1024
    e.d_length, e.d_budget, e.d_weight, e.d_weight_out, e.d_pos_out, e.d_length_out = range(0xa0000, 0x100000, 0x10000)
    return c, a, e


def call(lib, name, c, x):
    return getattr(lib, name)(ctypes.byref(c), ctypes.byref(x), None)


CACHE_FAULTS = [(dict(d_k=0), -1), (dict(d_v=0), -1), (dict(d_block_table=0), -1), (dict(d_k=0x10008), -2), (dict(d_status=0x40002), -2),
                (dict(n_seqs=-1), -3), (dict(n_blocks=0), -3), (dict(max_pages=0), -3), (dict(kv_heads=0), -3), (dict(reserved=1), -3),
                (dict(k_slot_stride=12), -3), (dict(v_block_stride=-8), -3), (dict(k_slot_stride=1 << 27), -3),
                (dict(v_head_stride=1 << 41), -3), (dict(dtype=2), -4), (dict(head_dim=96), -4), (dict(page_tokens=8), -4),
                (dict(page_tokens=48), -4), (dict(page_tokens=2048), -4)]
ATTENTION_FAULTS = [(dict(d_q=0), -1), (dict(d_out=0), -1), (dict(d_lse=0), -1), (dict(d_row_offset=0), -1), (dict(d_length=0), -1),
                    (dict(d_q=0x50004), -2), (dict(d_out=0x80008), -2), (dict(d_length=0x70001), -2), (dict(n_rows=-1), -3),
                    (dict(max_rows=-1), -3), (dict(max_len=1025), -3), (dict(max_len=-1), -3), (dict(q_heads=3), -3), (dict(q_heads=0), -3),
                    (dict(softcap=-1.0), -3), (dict(softcap=float("nan")), -3), (dict(softcap=float("inf")), -3),
                    (dict(scale=float("nan")), -3), (dict(q_row_stride=4), -3), (dict(out_head_stride=-8), -3), (dict(reserved=1), -3),
                    (dict(weight_seq_stride=-1), -3), (dict(d_parent=0x200000, max_rows=257), -4)]


@pytest.mark.parametrize("fault,status", CACHE_FAULTS)
def test_cache_checks(lib, fault, status):
    c, a, e = structs()
    for k, v in fault.items():
        setattr(c, k, v)
    a.d_weight = 0x300000
    for name, x in (("rkc_attend", a), ("rkc_weigh", a), ("rkc_evict", e)):
        assert call(lib, name, c, x) == status, name


@pytest.mark.parametrize("fault,status", ATTENTION_FAULTS)
def test_attention_checks(lib, fault, status):
    c, a, _ = structs()
    for k, v in fault.items():
        setattr(a, k, v)
    assert call(lib, "rkc_attend", c, a) == status
    a.d_weight = 0x300000
    if "d_out" not in fault:
        assert call(lib, "rkc_weigh", c, a) == status


def test_weigh_wants_an_account(lib):
    c, a, _ = structs()
    assert call(lib, "rkc_weigh", c, a) == -1
    a.d_weight = 0x300002
    assert call(lib, "rkc_weigh", c, a) == -2


@pytest.mark.parametrize("fault,status", [
    (dict(d_length=0), -1), (dict(d_budget=0), -1), (dict(d_weight=0), -1), (dict(d_weight_out=0), -1), (dict(d_pos_out=0), -1),
    (dict(d_length_out=0), -1), (dict(d_weight=0xc0001), -2), (dict(max_len=-1), -3), (dict(max_len=1025), -3), (dict(reserved=1), -3),
    (dict(weight_head_stride=-1), -3), (dict(d_weight_out=0xc0000), -3), (dict(d_pos=0xe0000), -3), (dict(d_length_out=0xa0000), -3)])
def test_eviction_checks(lib, fault, status):
    c, _, e = structs()
    for k, v in fault.items():
        setattr(e, k, v)
    assert call(lib, "rkc_evict", c, e) == status


def test_scratch(lib):
    null = None
    c, a, e = structs()
    c.max_pages, a.max_len = 256, 4096  # long enough that the attention splits a sequence
    for name, x in (("rkc_attend", a), ("rkc_evict", e)):
        need = getattr(lib, name + "_scratch_bytes")(ctypes.byref(c), ctypes.byref(x))
        assert need > 0
        assert call(lib, name, c, x) == -5
        x.scratch_bytes, x.d_scratch = need, 0x100080
        assert call(lib, name, c, x) == -2
        x.scratch_bytes, x.d_scratch = need - 1, 0x100000
        assert call(lib, name, c, x) == -5
        assert getattr(lib, name + "_scratch_bytes")(null, ctypes.byref(x)) == 0
        assert getattr(lib, name)(null, ctypes.byref(x), None) == -1
        assert getattr(lib, name)(ctypes.byref(c), None, None) == -1
    # nothing to do: fine without any buffer
    c.n_seqs = 0
    for f in ("d_k", "d_v", "d_block_table"):
        setattr(c, f, 0)
    a.d_q = a.d_out = 0
    for name, x in (("rkc_attend", a), ("rkc_weigh", a), ("rkc_evict", e)):
        assert call(lib, name, c, x) == 0


def test_scratch_is_bounded(lib):
    """Partial outputs of a split take at most a few MiB a CU, whatever the lengths."""
    for rows, length in ((1, 1 << 20), (64, 1 << 20), (4000, 1 << 16)):
        c, a, e = structs()
        c.max_pages = length // 16
        a.max_rows, a.max_len = rows, length
        n = lib.rkc_attend_scratch_bytes(ctypes.byref(c), ctypes.byref(a))
        assert n <= 256 * 4 * (1 << 20), (rows, length, n)


@pytest.mark.parametrize("name,what,fault", [
    ("rkc_attend", "a", dict(out_row_stride=0)), ("rkc_attend", "a", dict(out_head_stride=0)), ("rkc_attend", "a", dict(out_head_stride=120)),
    ("rkc_attend", "a", dict(out_row_stride=512)), ("rkc_attend", "a", dict(weight_seq_stride=0)),
    ("rkc_weigh", "a", dict(weight_head_stride=0)), ("rkc_weigh", "a", dict(weight_seq_stride=1024)), ("rkc_weigh", "a", dict(weight_head_stride=1000)),
    ("rkc_evict", "e", dict(weight_seq_stride=0)), ("rkc_evict", "e", dict(weight_head_stride=8)), ("rkc_evict", "c", dict(k_head_stride=0)),
    ("rkc_evict", "c", dict(v_block_stride=0)), ("rkc_evict", "c", dict(v_slot_stride=128)), ("rkc_evict", "e", dict(d_length_out=0xb0000)),
    ("rkc_evict", "e", dict(d_protect=0xf0000)), ("rkc_evict", "e", dict(d_recent_from=0xf0000))])
def test_outputs_keep_apart(lib, name, what, fault):
    """Elements that share memory are refused where a call writes them (-3); else the next thing wrong is the scratch."""
    c, a, e = structs()
    a.d_weight = 0x300000
    c.max_pages, a.max_len = 64, 1024
    x = e if name == "rkc_evict" else a
    for k, v in fault.items():
        setattr(dict(c=c, a=a, e=e)[what], k, v)
    assert call(lib, name, c, x) == -3


def test_orders_of_dimensions_keep_apart(lib):
    """Any order of the dimensions is fine, and so is the stride of a dimension of one; keys that are only read may be
    shared by the heads (the scratch is what is refused)."""
    c, a, e = structs()
    e.weight_seq_stride, e.weight_head_stride = 1024, 4096
    c.k_head_stride, c.k_block_stride, c.k_slot_stride = 300 * 16 * 128, 16 * 128, 128
    assert call(lib, "rkc_evict", c, e) == -5
    c.max_pages, a.max_len = 256, 4096
    a.out_row_stride, a.out_head_stride, c.k_head_stride = 128, 512, 0
    assert call(lib, "rkc_attend", c, a) == -5
    c.n_seqs = c.kv_heads = 1
    e.weight_seq_stride = e.weight_head_stride = 0
    c.v_head_stride = c.k_head_stride = 0
    c.max_pages = 64
    assert call(lib, "rkc_evict", c, e) == -5
