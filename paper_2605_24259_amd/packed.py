"""A paged KV cache in 4 bits -- Python binding of ``include/rkc_packed.h``.

A claim that is demoted, or a batch too large for the pool, can be held in 17 bits for each 64 of a 16-bit cache::

    pool = PackedCache.pool(blocks, page_tokens, kv_heads, head_dim)
    cache = PackedCache(pool, block_table, page_tokens=16, head_dim=128, dtype=torch.bfloat16)
    q = cache.store(k, v, row_offset, length, q=q, k_norm=..., q_norm=..., freq=...)   # rounded as they are written
    out, lse = cache.attend(q, row_offset, length, max_rows=n)
    k, v = cache.read(row_offset, length, rows=n)                                        # back to 16 bits

The 4 bits are those of the microscaling formats: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, times a power of two for
each 32 elements of a head.  A head's slot whose key or value has an element that is not finite reads back as NaN.  As with
``PagedCache``, nothing waits for the GPU, and there are no gradients.
"""
from __future__ import annotations

import ctypes
import math

from .cache import _Attention, _Cache, _Cached
from .rows import _Rows


class _Packed(ctypes.Structure):
    """rkc_packed (include/rkc_packed.h)."""
    _fields_ = [(n, ctypes.c_int32) for n in ("n_seqs", "n_blocks", "max_pages", "page_tokens", "kv_heads", "head_dim",
                                              "dtype", "reserved")]
    _fields_ += [(n, ctypes.c_int64) for n in ("block_stride", "head_stride")]
    _fields_ += [(n, ctypes.c_void_p) for n in ("d_pool", "d_block_table", "d_status")]


PACKED_EXPORTS = ("rkc_store", "rkc_read", "rkc_packed_store", "rkc_packed_read", "rkc_packed_attend_scratch_bytes", "rkc_packed_attend")


def declare(lib):
    """Argument and result types of the functions of include/rkc_packed.h."""
    c, p, r, a = (ctypes.POINTER(x) for x in (_Cache, _Packed, _Rows, _Attention))
    vp = ctypes.c_void_p
    for name, args in (("rkc_store", [c, r, vp]), ("rkc_read", [c, r, vp]), ("rkc_packed_store", [p, r, vp]),
                       ("rkc_packed_read", [p, r, vp]), ("rkc_packed_attend", [p, a, vp])):
        getattr(lib, name).argtypes, getattr(lib, name).restype = args, ctypes.c_int
    lib.rkc_packed_attend_scratch_bytes.argtypes, lib.rkc_packed_attend_scratch_bytes.restype = [p, a], ctypes.c_size_t


class PackedCache(_Cached):
    """Blocks of keys and values in 4 bits, and the sequences that lie in them.  Calls run on the current device, which has
    to be the cache's.

    pool         [blocks, kv_heads, page_tokens * (head_dim + head_dim / 16)] uint8 on the GPU, the last dimension contiguous,
                 strides and address multiples of 16 (``PackedCache.pool`` makes one): keys, values, the keys' scales and the
                 values' scales of a block's head, each [slots, ...]
    block_table  [seqs, pages] int32: the blocks of each sequence in order
    page_tokens  slots of a block: 16, 32, ... 1,024
    head_dim     64, 128 or 256
    dtype        bfloat16 or float16: of the rows that are stored and read, of queries and outputs
    status       [seqs] int32, as of ``PagedCache``
    """

    @staticmethod
    def pool(blocks, page_tokens, kv_heads, head_dim, device="cuda"):
        """A pool of zeros."""
        import torch
        return torch.zeros(blocks, kv_heads, page_tokens * (head_dim + head_dim // 16), dtype=torch.uint8, device=device)

    def __init__(self, pool, block_table, *, page_tokens, head_dim, dtype):
        import torch

        from . import load
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU: the operators run only in the HIP kernels")
        self._lib = load()
        types = {torch.bfloat16: 0, torch.float16: 1}
        if dtype not in types:
            raise TypeError(f"dtype: bfloat16 or float16 is wanted, got {dtype}")
        if pool.dtype is not torch.uint8 or pool.dim() != 3 or pool.shape[2] != page_tokens * (head_dim + head_dim // 16) or pool.stride(2) != 1:
            raise ValueError(f"pool: [blocks, kv_heads, {page_tokens * (head_dim + head_dim // 16)}] of uint8, the last dimension "
                             f"contiguous, is wanted, got {pool.dtype} {tuple(pool.shape)}")
        if not pool.is_cuda:
            raise ValueError("pool must be on a GPU")
        self._bind(torch, pool, block_table)
        self.pool, self.dtype, self._scale = pool, dtype, 1 / math.sqrt(head_dim)
        c = _Packed()
        c.n_seqs, c.max_pages = block_table.shape
        c.n_blocks, c.kv_heads, _ = pool.shape
        c.page_tokens, c.head_dim, c.dtype = page_tokens, head_dim, types[dtype]
        c.block_stride = pool.stride(0) if c.n_blocks > 1 else 0
        c.head_stride = pool.stride(1) if c.kv_heads > 1 else 0
        c.d_pool, c.d_block_table, c.d_status = pool.data_ptr(), block_table.data_ptr(), self.status.data_ptr()
        self._finish(c, self._lib.rkc_packed_store, self._lib.rkc_packed_read)

    def attend(self, q, row_offset, length, *, max_rows, max_len=None, scale=None, softcap=0.0, slope=None, prefix=None,
               row_start=None, parent=None, out=None, stream=None):
        """Attention of new rows, whose own keys and values are in the last slots of their sequences already: as
        ``PagedCache.attend``, over the values that the 4 bits stand for.  Returns (out, lse).  As there, the softmax's weights are
        rounded to the cache's type where more than 16 rows (``max_rows`` times the query heads of a key/value head) share a key."""
        head, q_strides, tail = self._attention(q, row_offset, length, max_rows, max_len, scale, softcap, slope, prefix, row_start, parent)
        if stream is not None:
            with self._on(stream):
                return self._run_attend(q, head, q_strides, tail, out, stream)
        return self._run_attend(q, head, q_strides, tail, out, None)

    def _run_attend(self, q, head, q_strides, tail, out, stream):
        out, lse = self._outputs(q, out)
        a = _Attention(*head, 1.0, 0, *q_strides, out.stride(0), out.stride(1), 0, 0, *tail, out.data_ptr(), lse.data_ptr())
        ref = ctypes.byref(a)
        need = self._lib.rkc_packed_attend_scratch_bytes(self._c_ref, ref)
        if need:
            scratch = self._scratch(need)
            a.d_scratch, a.scratch_bytes = scratch.data_ptr(), need
        self._call(self._lib.rkc_packed_attend, "rkc_packed_attend", ref, stream)
        return out, lse
