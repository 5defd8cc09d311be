"""Operators on the contents of a paged KV cache -- Python binding of ``include/rkc_cache.h``.

The replay decides what happens to a pool's blocks; a ``PagedCache`` works on what they hold::

    cache = PagedCache(k, v, block_table)        # [blocks, slots, kv_heads, head_dim], [seqs, pages]
    out, lse = cache.attend(q, row_offset, length, max_rows=n)              # a prompt's chunk
    out, lse = cache.attend(q, row_offset, length, max_rows=n, parent=p)    # a tree of drafted tokens
    weight = cache.weigh(q, lse, row_offset, length, max_rows=n)            # the account of the slots
    length, weight, pos = cache.evict(weight, length, budget, protect=claimed)

Everything runs in the library's HIP kernels on the current stream (or ``stream``); torch provides buffers.
Nothing is copied to the host and no call waits for the GPU.  The operators are for serving: they have no gradients, and
what they return has no history, also where queries or a cache require one.
"""
from __future__ import annotations

import contextlib
import ctypes
import math

from . import RkcError, _stream_ptr

MAX_TREE_ROWS = 256
HEAD_DIMS = (64, 128, 256)
# bits of ``PagedCache.status`` (rkc_cache_status)
CS_LENGTH, CS_BLOCK, CS_PARENT = 1, 2, 4


class _Cache(ctypes.Structure):
    """rkc_cache (include/rkc_cache.h)."""
    _fields_ = [(n, ctypes.c_int32) for n in ("n_seqs", "n_blocks", "max_pages", "page_tokens", "kv_heads", "head_dim",
                                              "dtype", "reserved")]
    _fields_ += [(n, ctypes.c_int64) for n in ("k_block_stride", "k_slot_stride", "k_head_stride", "v_block_stride",
                                               "v_slot_stride", "v_head_stride")]
    _fields_ += [(n, ctypes.c_void_p) for n in ("d_k", "d_v", "d_block_table", "d_status")]


class _Attention(ctypes.Structure):
    """rkc_attention."""
    _fields_ = [(n, ctypes.c_int32) for n in ("n_rows", "q_heads", "max_rows", "max_len")]
    _fields_ += [(n, ctypes.c_float) for n in ("scale", "softcap", "decay")]
    _fields_ += [("reserved", ctypes.c_int32)]
    _fields_ += [(n, ctypes.c_int64) for n in ("q_row_stride", "q_head_stride", "out_row_stride", "out_head_stride",
                                               "weight_seq_stride", "weight_head_stride")]
    _fields_ += [(n, ctypes.c_void_p) for n in ("d_q", "d_row_offset", "d_length", "d_row_start", "d_prefix", "d_parent",
                                                "d_slope", "d_out", "d_lse", "d_weight_in", "d_weight", "d_scratch")]
    _fields_ += [("scratch_bytes", ctypes.c_size_t)]


class _Eviction(ctypes.Structure):
    """rkc_eviction."""
    _fields_ = [(n, ctypes.c_int32) for n in ("max_len", "reserved")]
    _fields_ += [(n, ctypes.c_int64) for n in ("weight_seq_stride", "weight_head_stride")]
    _fields_ += [(n, ctypes.c_void_p) for n in ("d_length", "d_budget", "d_protect", "d_recent_from", "d_weight", "d_pos",
                                                "d_weight_out", "d_pos_out", "d_length_out", "d_scratch")]
    _fields_ += [("scratch_bytes", ctypes.c_size_t)]


CACHE_EXPORTS = ("rkc_attend_scratch_bytes", "rkc_evict_scratch_bytes", "rkc_attend", "rkc_weigh", "rkc_evict")


def declare(lib):
    """Argument and result types of the functions here."""
    c, a, e, vp = ctypes.POINTER(_Cache), ctypes.POINTER(_Attention), ctypes.POINTER(_Eviction), ctypes.c_void_p
    for name, args in (("rkc_attend_scratch_bytes", [c, a]), ("rkc_evict_scratch_bytes", [c, e])):
        getattr(lib, name).argtypes, getattr(lib, name).restype = args, ctypes.c_size_t
    for name, args in (("rkc_attend", [c, a, vp]), ("rkc_weigh", [c, a, vp]), ("rkc_evict", [c, e, vp])):
        getattr(lib, name).argtypes, getattr(lib, name).restype = args, ctypes.c_int


_HERE = contextlib.nullcontext()


class PagedCache:
    """Blocks of keys and values, and the sequences that lie in them.  Calls run on the current device, which has to be
    the cache's.

    k, v         [blocks, slots, kv_heads, head_dim], bfloat16 or float16, on the GPU: any strides (multiples of 8
                 elements) with the last dimension contiguous; 16, 32, ... 1,024 slots a block; head_dim 64, 128 or
                 256.  ``evict`` moves rows of them in place.
    block_table  [seqs, pages] int32: the blocks of each sequence in order
    status       [seqs] int32, zeros at first: CS_* bits of what calls found wrong in device memory (lengths, block
                 ids, parents); the user clears it
    """

    def __init__(self, k, v, block_table):
        import torch

        from . import load
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU: the operators run only in the HIP kernels")
        self._lib = load()
        types = {torch.bfloat16: 0, torch.float16: 1}
        if k.dim() != 4 or k.shape != v.shape:
            raise ValueError(f"k and v are [blocks, slots, kv_heads, head_dim], alike: {tuple(k.shape)}, {tuple(v.shape)}")
        if k.dtype not in types or v.dtype != k.dtype:
            raise TypeError(f"k and v are bfloat16 or float16, alike: {k.dtype}, {v.dtype}")
        if k.stride(3) != 1 or v.stride(3) != 1:
            raise ValueError("the last dimension of k and v must be contiguous")
        self._int32, self._torch, self._raw_stream = torch.int32, torch, torch._C._cuda_getCurrentRawStream
        self._index, self._scale = k.get_device(), 1 / math.sqrt(k.shape[3])
        self.k, self.v, self.device, self.dtype = k, v, k.device, k.dtype
        if not k.is_cuda or v.device != k.device:
            raise ValueError("k and v must be on one GPU")
        if block_table.dtype is not torch.int32 or block_table.device != self.device or block_table.dim() != 2 or \
                not block_table.is_contiguous():
            raise ValueError(f"block_table: a contiguous int32 tensor [seqs, pages] on {self.device} is wanted")
        self.block_table = block_table
        self.status = torch.zeros(block_table.shape[0], dtype=torch.int32, device=self.device)
        c = _Cache()
        c.n_seqs, c.max_pages = block_table.shape
        c.n_blocks, c.page_tokens, c.kv_heads, c.head_dim = k.shape
        c.dtype = types[k.dtype]
        c.k_block_stride, c.k_slot_stride, c.k_head_stride = k.stride()[:3]
        c.v_block_stride, c.v_slot_stride, c.v_head_stride = v.stride()[:3]
        c.d_k, c.d_v, c.d_block_table, c.d_status = k.data_ptr(), v.data_ptr(), block_table.data_ptr(), self.status.data_ptr()
        self._c, self._c_ref = c, ctypes.byref(c)
        self.n_seqs, self.kv_heads, self.head_dim = int(c.n_seqs), int(c.kv_heads), int(c.head_dim)
        self.max_len = int(c.max_pages) * int(c.page_tokens)

    def _ints(self, t, name, n):
        """Address of a contiguous int32 tensor of n values on the cache's device."""
        if t.dtype is not self._int32 or t.get_device() != self._index or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
            raise ValueError(f"{name}: a contiguous int32 tensor of {n} values on {self.device} is wanted, got {t.dtype} "
                             f"{tuple(t.shape)} on {t.device}")
        return t.data_ptr()

    def _account(self, t, name, dtype, max_len):
        """Strides of an account (or of its positions)."""
        if t.dtype is not dtype or t.get_device() != self._index or t.dim() != 3 or \
                t.shape[0] != self.n_seqs or t.shape[1] != self.kv_heads or t.shape[2] < max_len or t.stride(2) != 1:
            raise ValueError(f"{name}: [{self.n_seqs}, {self.kv_heads}, >= {max_len}] of {dtype} on {self.device}, the last "
                             f"dimension contiguous, is wanted, got {t.dtype} {tuple(t.shape)} on {t.device}")
        # of a dimension of one, the stride says nothing
        return t.stride(0) if self.n_seqs > 1 else 0, t.stride(1) if self.kv_heads > 1 else 0

    def _attention(self, q, row_offset, length, max_rows, max_len, scale, softcap, slope, prefix, row_start, parent):
        """Checks what attend and weigh share; the fields of rkc_attention in two runs, around those of the outputs."""
        if q.dim() != 3 or q.shape[2] != self.head_dim or q.dtype is not self.dtype or q.get_device() != self._index or q.stride(2) != 1:
            raise ValueError(f"q: [rows, heads, {self.head_dim}] of {self.dtype} on {self.device}, the last dimension "
                             f"contiguous, is wanted, got {q.dtype} {tuple(q.shape)} on {q.device}")
        n, heads, _ = q.shape
        if heads % self.kv_heads or not heads:
            raise ValueError(f"q: {heads} heads are no multiple of the cache's {self.kv_heads}")
        if slope is not None and (slope.dtype is not self._torch.float32 or slope.get_device() != self._index
                                  or not slope.is_contiguous() or tuple(slope.shape) != (heads,)):
            raise ValueError(f"slope: [{heads}] float32 on {self.device} is wanted")
        offsets, lengths = self._ints(row_offset, "row_offset", self.n_seqs + 1), self._ints(length, "length", self.n_seqs)
        head = (n, heads, max_rows, self.max_len if max_len is None else max_len, self._scale if scale is None else scale, softcap)
        tail = (q.data_ptr(), offsets, lengths, None if row_start is None else self._ints(row_start, "row_start", n),
                None if prefix is None else self._ints(prefix, "prefix", self.n_seqs),
                None if parent is None else self._ints(parent, "parent", n), None if slope is None else slope.data_ptr())
        return head, (q.stride(0), q.stride(1)), tail

    def _weights(self, weight, weight_out, n):
        """(weight_out, its strides) for the account `weight`, or none."""
        torch = self._torch
        at = None if weight is None else self._account(weight, "weight", torch.float32, n)
        if weight_out is None:
            weight_out = torch.zeros(self.n_seqs, self.kv_heads, n, device=self.device) if weight is None else \
                torch.empty_strided(weight.shape, weight.stride(), dtype=weight.dtype, device=self.device).zero_()
        to = self._account(weight_out, "weight_out", torch.float32, n)
        if at is not None and at != to:
            raise ValueError(f"weight and weight_out differ in strides: {weight.stride()}, {weight_out.stride()}")
        return weight_out, to

    def _call(self, f, name, args, stream):
        # the current stream of the cache's device; looked up by number, a twentieth of the cost of a Stream object
        st = f(self._c_ref, args, self._raw_stream(self._index) if stream is None else _stream_ptr(stream))
        if st != 0:
            raise RkcError(st, name)

    def _on(self, stream):
        """Tensors made in a call belong to the stream that the call runs on."""
        return _HERE if stream is None else self._torch.cuda.stream(stream)

    def _scratch(self, need):
        return self._torch.empty(need, dtype=self._torch.uint8, device=self.device)

    def attend(self, q, row_offset, length, *, max_rows, max_len=None, scale=None, softcap=0.0, slope=None, prefix=None,
               row_start=None, parent=None, out=None, weight=None, decay=1.0, weight_out=None, stream=None):
        """Attention of new rows, whose own keys and values are in the last slots of their sequences already.

        q           [rows, heads, head_dim] of the cache's type; heads a multiple of kv_heads
        row_offset  [seqs + 1] int32: sequence s has rows row_offset[s] .. row_offset[s + 1]
        length      [seqs] int32: slots of each sequence, the rows' own among them
        max_rows    >= every sequence's rows; with ``parent`` at most 256
        max_len     >= every length (default: what the block table holds); the smaller, the better the split
        softcap     > 0: scores become softcap * tanh(score / softcap)
        slope       [heads] float32: scores lose slope * distance
        prefix      [seqs] int32: leading slots that every row sees
        row_start   [rows] int32: the first slot a row sees beside the prefix (its document's start)
        parent      [rows] int32: rows are a tree; a row's parent within its sequence, -1 for a root
        weight      with it or ``weight_out``: the rows' attention weights are added to the account as in ``weigh``
        out         takes the outputs; may be q where there is no account

        Returns (out, lse), or (out, lse, weight_out): out as q, lse [rows, heads] float32, the natural logarithm
        of the softmax sums.  A row that sees nothing gets zeros and -inf.
        """
        head, q_strides, tail = self._attention(q, row_offset, length, max_rows, max_len, scale, softcap, slope, prefix, row_start, parent)
        weigh, strides = weight is not None or weight_out is not None, (0, 0)
        with self._on(stream):
            if out is None:
                out = q.new_empty(q.shape)
            elif out.shape != q.shape or out.dtype is not q.dtype or out.get_device() != self._index or out.stride(2) != 1:
                raise ValueError("out: a tensor like q, the last dimension contiguous, is wanted")
            lse = q.new_empty(q.shape[:2], dtype=self._torch.float32)
            if weigh:
                weight_out, strides = self._weights(weight, weight_out, head[3])
            a = _Attention(*head, decay, 0, *q_strides, out.stride(0), out.stride(1), *strides, *tail, out.data_ptr(), lse.data_ptr(),
                           None if weight is None else weight.data_ptr(), weight_out.data_ptr() if weigh else None)
            ref = ctypes.byref(a)
            need = self._lib.rkc_attend_scratch_bytes(self._c_ref, ref)
            if need:
                scratch = self._scratch(need)
                a.d_scratch, a.scratch_bytes = scratch.data_ptr(), need
            self._call(self._lib.rkc_attend, "rkc_attend", ref, stream)
        return (out, lse, weight_out) if weigh else (out, lse)

    def weigh(self, q, lse, row_offset, length, *, max_rows, max_len=None, scale=None, softcap=0.0, slope=None, prefix=None,
              row_start=None, parent=None, weight=None, decay=1.0, weight_out=None, stream=None):
        """Adds the attention weights of rows to the account of their sequences' slots.

        q, row_offset, length and what follows as in ``attend``; lse as it returned it.  Slot j of key/value head h
        gets  decay * weight[s, h, j] + sum of exp(score - lse)  over the rows and the head's queries; slots behind
        the length are left alone.  weight_out may be weight; by default it is new and zero behind the length.
        """
        head, q_strides, tail = self._attention(q, row_offset, length, max_rows, max_len, scale, softcap, slope, prefix, row_start, parent)
        if lse.dtype is not self._torch.float32 or lse.shape != q.shape[:2] or lse.get_device() != self._index or not lse.is_contiguous():
            raise ValueError(f"lse: a contiguous float32 tensor {tuple(q.shape[:2])} on {self.device} is wanted")
        with self._on(stream):
            weight_out, strides = self._weights(weight, weight_out, head[3])
            a = _Attention(*head, decay, 0, *q_strides, 0, 0, *strides, *tail, None, lse.data_ptr(),
                           None if weight is None else weight.data_ptr(), weight_out.data_ptr())
            self._call(self._lib.rkc_weigh, "rkc_weigh", ctypes.byref(a), stream)
        return weight_out

    def evict(self, weight, length, budget, *, protect=None, recent_from=None, pos=None, max_len=None, weight_out=None,
              pos_out=None, stream=None):
        """Brings sequences down to min(length, max(budget, protect)) slots, head by head.

        weight       [seqs, kv_heads, >= max_len] float32: the account; the larger stays, ties: the lower slot
        budget       [seqs] int32: slots to keep
        protect      [seqs] int32: leading slots that stay in place (those of a resident claim, or shared ones)
        pos          as weight, int32: positions of the slots' tokens (default: the slots' numbers)
        recent_from  [seqs] int32: slots of this position or a later one go before the others

        What is kept behind the new end moves into the gaps before it (in order); keys and values change in place, and
        the blocks behind the new length are free.  Returns (length, weight_out, pos_out) as new tensors (or the
        ones given), valid up to the new lengths.
        """
        torch = self._torch
        n = min(self.max_len, weight.shape[-1]) if max_len is None else max_len
        strides = self._account(weight, "weight", torch.float32, n)
        with self._on(stream):
            if weight_out is None:
                weight_out = torch.empty_strided(weight.shape, weight.stride(), dtype=weight.dtype, device=self.device)
            if pos_out is None:
                pos_out = torch.empty_strided(weight.shape, weight.stride(), dtype=torch.int32, device=self.device)
            for name, t, dtype in (("weight_out", weight_out, torch.float32), ("pos", pos, torch.int32), ("pos_out", pos_out, torch.int32)):
                if t is not None and self._account(t, name, dtype, n) != strides:
                    raise ValueError(f"{name} and weight differ in strides: {t.stride()}, {weight.stride()}")
            length_out = torch.empty_like(length)
            e = _Eviction(n, 0, *strides, self._ints(length, "length", self.n_seqs), self._ints(budget, "budget", self.n_seqs),
                          None if protect is None else self._ints(protect, "protect", self.n_seqs),
                          None if recent_from is None else self._ints(recent_from, "recent_from", self.n_seqs),
                          weight.data_ptr(), None if pos is None else pos.data_ptr(), weight_out.data_ptr(), pos_out.data_ptr(),
                          length_out.data_ptr())
            ref = ctypes.byref(e)
            need = self._lib.rkc_evict_scratch_bytes(self._c_ref, ref)
            scratch = self._scratch(need)
            e.d_scratch, e.scratch_bytes = scratch.data_ptr(), need
            self._call(self._lib.rkc_evict, "rkc_evict", ref, stream)
        return length_out, weight_out, pos_out
