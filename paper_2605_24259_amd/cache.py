"""Operators on the contents of a paged KV cache -- Python binding of ``include/rkc_cache.h``.

The replay decides what happens to a pool's blocks; a ``PagedCache`` works on what they hold::

    cache = PagedCache(k, v, block_table)        # [blocks, slots, kv_heads, head_dim], [seqs, pages]
    out, lse = cache.attend(q, row_offset, length, max_rows=n)              # a prompt's chunk
    out, lse = cache.attend(q, row_offset, length, max_rows=n, parent=p)    # a tree of drafted tokens
    weight = cache.weigh(q, lse, row_offset, length, max_rows=n)            # the account of the slots
    length, weight, pos = cache.evict(weight, length, budget, protect=claimed)

Everything runs in the library's HIP kernels on the current stream (or ``stream``); torch provides buffers.
Nothing is copied to the host and no call waits for the GPU.
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


def _ptr(t):
    return t.data_ptr() if t is not None else None


class PagedCache:
    """Blocks of keys and values, and the sequences that lie in them.

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
        self._int32 = torch.int32
        self.k, self.v, self.device, self.dtype = k, v, k.device, k.dtype
        if not k.is_cuda or v.device != k.device:
            raise ValueError("k and v must be on one GPU")
        self.block_table = self._ints(block_table, "block_table", 2)
        self.status = torch.zeros(block_table.shape[0], dtype=torch.int32, device=self.device)
        c = _Cache()
        c.n_seqs, c.max_pages = block_table.shape
        c.n_blocks, c.page_tokens, c.kv_heads, c.head_dim = k.shape
        c.dtype = types[k.dtype]
        c.k_block_stride, c.k_slot_stride, c.k_head_stride = k.stride()[:3]
        c.v_block_stride, c.v_slot_stride, c.v_head_stride = v.stride()[:3]
        c.d_k, c.d_v, c.d_block_table, c.d_status = k.data_ptr(), v.data_ptr(), _ptr(self.block_table), _ptr(self.status)
        self._c, self._c_ref = c, ctypes.byref(c)
        self._torch, self._raw_stream = torch, torch._C._cuda_getCurrentRawStream
        self._index = k.device.index
        self.n_seqs, self.kv_heads, self.head_dim = int(c.n_seqs), int(c.kv_heads), int(c.head_dim)
        self.max_len = int(c.max_pages) * int(c.page_tokens)

    def _ints(self, t, name, dim=1, n=None, optional=False):
        if t is None and optional:
            return None
        if t.dtype != self._int32 or t.device != self.device or t.dim() != dim or not t.is_contiguous():
            raise ValueError(f"{name}: a contiguous int32 tensor of {dim} dimension(s) on {self.device} is wanted")
        if n is not None and t.shape[0] != n:
            raise ValueError(f"{name}: {n} values are wanted, got {t.shape[0]}")
        return t

    def _account(self, t, name, dtype, max_len):
        if t.dtype != dtype or t.device != self.device or t.dim() != 3 or t.stride(2) != 1 or \
                t.shape[0] != self.n_seqs or t.shape[1] != self.kv_heads or t.shape[2] < max_len:
            raise ValueError(f"{name}: [{self.n_seqs}, {self.kv_heads}, >= {max_len}] of {dtype} on {self.device}, the last "
                             "dimension contiguous, is wanted")
        return t

    def _attention(self, q, row_offset, length, max_rows, max_len, scale, softcap, slope, prefix, row_start, parent):
        torch = self._torch
        if q.dim() != 3 or q.shape[2] != self.head_dim or q.dtype != self.dtype or q.device != self.device or q.stride(2) != 1:
            raise ValueError(f"q: [rows, heads, {self.head_dim}] of {self.dtype} on {self.device}, the last dimension "
                             "contiguous, is wanted")
        if q.shape[1] % self.kv_heads or not q.shape[1]:
            raise ValueError(f"q: {q.shape[1]} heads are no multiple of the cache's {self.kv_heads}")
        n = q.shape[0]
        if slope is not None and (slope.dtype != torch.float32 or slope.device != self.device or not slope.is_contiguous()
                                  or tuple(slope.shape) != (q.shape[1],)):
            raise ValueError(f"slope: [{q.shape[1]}] float32 on {self.device} is wanted")
        a = _Attention()
        a.n_rows, a.q_heads, a.max_rows = n, q.shape[1], max_rows
        a.max_len = self.max_len if max_len is None else max_len
        a.scale = 1 / math.sqrt(self.head_dim) if scale is None else scale
        a.softcap, a.decay = softcap, 1.0
        a.q_row_stride, a.q_head_stride = q.stride(0), q.stride(1)
        a.d_q = q.data_ptr()
        a.d_row_offset = _ptr(self._ints(row_offset, "row_offset", n=self.n_seqs + 1))
        a.d_length = _ptr(self._ints(length, "length", n=self.n_seqs))
        a.d_row_start = _ptr(self._ints(row_start, "row_start", n=n, optional=True))
        a.d_prefix = _ptr(self._ints(prefix, "prefix", n=self.n_seqs, optional=True))
        a.d_parent = _ptr(self._ints(parent, "parent", n=n, optional=True))
        a.d_slope = _ptr(slope)
        return a

    def _weights(self, a, weight, weight_out, decay):
        torch = self._torch
        n = int(a.max_len)
        if weight is not None:
            self._account(weight, "weight", torch.float32, n)
        if weight_out is None:
            weight_out = torch.zeros(self.n_seqs, self.kv_heads, n, device=self.device) if weight is None else \
                torch.empty_strided(weight.shape, weight.stride(), dtype=weight.dtype, device=self.device).zero_()
        else:
            self._account(weight_out, "weight_out", torch.float32, n)
        if weight is not None and weight.stride() != weight_out.stride():
            raise ValueError(f"weight and weight_out differ in strides: {weight.stride()}, {weight_out.stride()}")
        a.weight_seq_stride, a.weight_head_stride = weight_out.stride()[:2]
        a.d_weight_in, a.d_weight, a.decay = _ptr(weight), weight_out.data_ptr(), decay
        return weight_out

    def _call(self, name, args, stream):
        # the current stream of the cache's device; looked up by number, a twentieth of the cost of a Stream object
        at = self._raw_stream(self._index) if stream is None else _stream_ptr(stream)
        st = getattr(self._lib, name)(self._c_ref, ctypes.byref(args), at)
        if st != 0:
            raise RkcError(st, name)

    def _on(self, stream):
        """Tensors made in a call belong to the stream that the call runs on."""
        return self._torch.cuda.stream(stream) if stream is not None else _HERE

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

        Returns (out, lse), or (out, lse, weight_out): out as q, lse [rows, heads] float32, the natural logarithm
        of the softmax sums.  A row that sees nothing gets zeros and -inf.
        """
        torch = self._torch
        a = self._attention(q, row_offset, length, max_rows, max_len, scale, softcap, slope, prefix, row_start, parent)
        with self._on(stream):
            if out is None:
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            elif out.shape != q.shape or out.dtype != q.dtype or out.device != q.device or out.stride(2) != 1:
                raise ValueError("out: a tensor like q, the last dimension contiguous, is wanted")
            lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
            a.out_row_stride, a.out_head_stride = out.stride(0), out.stride(1)
            a.d_out, a.d_lse = out.data_ptr(), lse.data_ptr()
            weigh = weight is not None or weight_out is not None
            if weigh:
                weight_out = self._weights(a, weight, weight_out, decay)
            need = self._lib.rkc_attend_scratch_bytes(self._c_ref, ctypes.byref(a))
            if need:
                scratch = torch.empty(need, dtype=torch.uint8, device=q.device)
                a.d_scratch, a.scratch_bytes = scratch.data_ptr(), need
            self._call("rkc_attend", a, stream)
        return (out, lse, weight_out) if weigh else (out, lse)

    def weigh(self, q, lse, row_offset, length, *, max_rows, max_len=None, scale=None, softcap=0.0, slope=None, prefix=None,
              row_start=None, parent=None, weight=None, decay=1.0, weight_out=None, stream=None):
        """Adds the attention weights of rows to the account of their sequences' slots.

        q, row_offset, length and what follows as in ``attend``; lse as it returned it.  Slot j of key/value head h
        gets  decay * weight[s, h, j] + sum of exp(score - lse)  over the rows and the head's queries; slots behind
        the length are left alone.  weight_out may be weight; by default it is new and zero behind the length.
        """
        torch = self._torch
        a = self._attention(q, row_offset, length, max_rows, max_len, scale, softcap, slope, prefix, row_start, parent)
        if lse.dtype != torch.float32 or lse.shape != q.shape[:2] or lse.device != self.device or not lse.is_contiguous():
            raise ValueError(f"lse: a contiguous float32 tensor {tuple(q.shape[:2])} on {self.device} is wanted")
        a.d_lse = lse.data_ptr()
        with self._on(stream):
            weight_out = self._weights(a, weight, weight_out, decay)
            self._call("rkc_weigh", a, stream)
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
        n = (min(self.max_len, weight.shape[-1]) if max_len is None else max_len)
        self._account(weight, "weight", torch.float32, n)
        e = _Eviction()
        with self._on(stream):
            if weight_out is None:
                weight_out = torch.empty_strided(weight.shape, weight.stride(), dtype=weight.dtype, device=self.device)
            if pos_out is None:
                pos_out = torch.empty_strided(weight.shape, weight.stride(), dtype=torch.int32, device=self.device)
            self._account(weight_out, "weight_out", torch.float32, n)
            for name, t in (("pos", pos), ("pos_out", pos_out)):
                if t is not None:
                    self._account(t, name, torch.int32, n)
            for name, t in (("weight_out", weight_out), ("pos", pos), ("pos_out", pos_out)):
                if t is not None and t.stride() != weight.stride():
                    raise ValueError(f"{name} and weight differ in strides: {t.stride()}, {weight.stride()}")
            e.max_len = n
            e.weight_seq_stride, e.weight_head_stride = weight.stride()[:2]
            e.d_length = _ptr(self._ints(length, "length", n=self.n_seqs))
            e.d_budget = _ptr(self._ints(budget, "budget", n=self.n_seqs))
            e.d_protect = _ptr(self._ints(protect, "protect", n=self.n_seqs, optional=True))
            e.d_recent_from = _ptr(self._ints(recent_from, "recent_from", n=self.n_seqs, optional=True))
            e.d_weight, e.d_pos = weight.data_ptr(), _ptr(pos)
            length_out = torch.empty_like(length)
            e.d_weight_out, e.d_pos_out, e.d_length_out = weight_out.data_ptr(), pos_out.data_ptr(), length_out.data_ptr()
            need = self._lib.rkc_evict_scratch_bytes(self._c_ref, ctypes.byref(e))
            scratch = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
            e.d_scratch, e.scratch_bytes = scratch.data_ptr(), scratch.numel()
            self._call("rkc_evict", e, stream)
        return length_out, weight_out, pos_out
