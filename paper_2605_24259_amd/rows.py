"""Rows into a paged KV cache and back -- Python binding of the stores and reads of ``include/rkc_packed.h``.

``RowOps`` gives ``store`` and ``read`` to both kinds of cache, ``PagedCache`` (16 bits) and ``PackedCache`` (4 bits).
"""
from __future__ import annotations

import ctypes

from . import RkcError, _stream_ptr

MAX_AXES = 8


class _Rows(ctypes.Structure):
    """rkc_rows (include/rkc_packed.h)."""
    _fields_ = [(n, ctypes.c_int32) for n in ("n_rows", "q_heads", "max_len", "n_freq", "axes", "interleaved", "norm_f32")]
    _fields_ += [("eps", ctypes.c_float)]
    _fields_ += [(n, ctypes.c_int64) for n in ("k_row_stride", "k_head_stride", "v_row_stride", "v_head_stride", "q_row_stride",
                                               "q_head_stride", "q_out_row_stride", "q_out_head_stride")]
    _fields_ += [(n, ctypes.c_void_p) for n in ("d_k", "d_v", "d_q", "d_q_out", "d_row_offset", "d_length", "d_position",
                                                "d_axis", "d_freq", "d_q_norm", "d_k_norm")]


class RowOps:
    """``store`` and ``read`` of a cache with the fields of ``PagedCache``; ``_store`` and ``_read`` name the library's
    functions."""

    _store, _read = "rkc_store", "rkc_read"

    def _heads_of(self, t, name, rows=None):
        """A tensor of rows: its strides, of a dimension of one 0, as they say nothing."""
        if t.dim() != 3 or t.shape[2] != self.head_dim or t.dtype is not self.dtype or t.get_device() != self._index or \
                t.stride(2) != 1 or (rows is not None and (t.shape[0] != rows or t.shape[1] != self.kv_heads)):
            raise ValueError(f"{name}: [{'rows' if rows is None else rows}, {'heads' if rows is None else self.kv_heads}, "
                             f"{self.head_dim}] of {self.dtype} on {self.device}, the last dimension contiguous, is wanted, got "
                             f"{t.dtype} {tuple(t.shape)} on {t.device}")
        n, h, _ = t.shape
        return t.stride(0) if n > 1 else 0, t.stride(1) if h > 1 else 0

    def _run_rows(self, f, r, stream):
        st = getattr(self._lib, f)(self._c_ref, ctypes.byref(r), self._raw_stream(self._index) if stream is None else _stream_ptr(stream))
        if st != 0:
            raise RkcError(st, f)

    def store(self, k, v, row_offset, length, *, q=None, q_norm=None, k_norm=None, eps=1e-6, freq=None, position=None, axis=None,
              interleaved=False, q_out=None, stream=None):
        """Puts keys and values of new rows into the last slots of their sequences, after the norm and the rotation of keys
        (and queries) where they are given: one pass over the rows.

        k, v        [rows, kv_heads, head_dim] of the cache's type; views of a fused projection are fine
        row_offset  [seqs + 1] int32: sequence s has rows row_offset[s] .. row_offset[s + 1]; no two rows may have one slot
        length      [seqs] int32: slots of each sequence, the rows' own among them
        q           [rows, heads, head_dim]: queries of the rows, any number of heads
        q_norm, k_norm  [head_dim] of the cache's type or float32 (both alike): heads are multiplied by
                    norm / sqrt(mean of squares + eps)
        freq        [pairs] float32, a multiple of 8 pairs up to head_dim / 2: pair j turns by freq[j] * position
        position    [rows] or [axes, rows] int32 (default: the rows' slots); up to 8 axes
        axis        [pairs] int32: the axis whose position a pair turns by (time, height, width); with more than one
        interleaved pairs are elements 2 j and 2 j + 1 instead of j and j + pairs
        q_out       takes the queries; may be q

        Returns the queries (q_out or a new tensor), or None without q.  A cache of 4 bits rounds keys and values as they
        are written; keys are computed in 64 bits up to that.
        """
        n, torch = k.shape[0], self._torch
        r = _Rows()
        r.k_row_stride, r.k_head_stride = self._heads_of(k, "k", n)
        r.v_row_stride, r.v_head_stride = self._heads_of(v, "v", n)
        r.n_rows, r.max_len, r.eps, r.interleaved, r.axes = n, self.max_len, eps, bool(interleaved), 1
        r.d_k, r.d_v = k.data_ptr(), v.data_ptr()
        r.d_row_offset, r.d_length = self._ints(row_offset, "row_offset", self.n_seqs + 1), self._ints(length, "length", self.n_seqs)
        if q_norm is not None or k_norm is not None:
            kind = (k_norm if q_norm is None else q_norm).dtype
            for t, name in ((q_norm, "q_norm"), (k_norm, "k_norm")):
                if t is not None and (t.dtype is not kind or (kind is not self.dtype and kind is not torch.float32) or t.get_device() != self._index
                                      or not t.is_contiguous() or tuple(t.shape) != (self.head_dim,)):
                    raise ValueError(f"{name}: a contiguous tensor [{self.head_dim}] of {self.dtype} or float32 (both norms alike) on "
                                     f"{self.device} is wanted, got {t.dtype} {tuple(t.shape)} on {t.device}")
            r.norm_f32 = kind is torch.float32
            r.d_q_norm = None if q_norm is None else q_norm.data_ptr()
            r.d_k_norm = None if k_norm is None else k_norm.data_ptr()
        if freq is not None:
            if freq.dtype is not torch.float32 or freq.get_device() != self._index or freq.dim() != 1 or not freq.is_contiguous() or \
                    freq.shape[0] % 8 or freq.shape[0] > self.head_dim // 2:
                raise ValueError(f"freq: a contiguous float32 tensor of 8, 16, ... {self.head_dim // 2} values on {self.device} is wanted, "
                                 f"got {freq.dtype} {tuple(freq.shape)} on {freq.device}")
            r.n_freq, r.d_freq = freq.shape[0], freq.data_ptr()
        if position is not None:
            if position.dtype is not torch.int32 or position.get_device() != self._index or not position.is_contiguous() or \
                    position.dim() not in (1, 2) or position.shape[-1] != n or (position.dim() == 2 and not 1 <= position.shape[0] <= MAX_AXES):
                raise ValueError(f"position: a contiguous int32 tensor [{n}] or [up to {MAX_AXES}, {n}] on {self.device} is wanted, got "
                                 f"{position.dtype} {tuple(position.shape)} on {position.device}")
            r.d_position = position.data_ptr()
            if position.dim() == 2:
                r.axes = position.shape[0]
        if axis is not None:
            if position is None or freq is None:
                raise ValueError("axis: there are several axes only of given positions and frequencies")
            r.d_axis = self._ints(axis, "axis", r.n_freq)
        elif r.axes > 1 and freq is not None:
            raise ValueError(f"position: of {r.axes} axes, axis has to say which one each of the {r.n_freq} pairs turns by")
        elif r.axes > 1:
            r.axes, r.d_position = 1, None  # nothing turns
        if q is None:
            if q_norm is not None or q_out is not None:
                raise ValueError("q_norm and q_out are of queries, and there are none")
        else:
            if q.shape[0] != n:
                raise ValueError(f"q: {q.shape[0]} rows, and {n} of k")
            r.q_row_stride, r.q_head_stride = self._heads_of(q, "q")
            with self._on(stream):
                if q_out is None:
                    q_out = q.new_empty(q.shape)
                elif q_out.shape != q.shape:
                    raise ValueError(f"q_out: {tuple(q_out.shape)}, and q is {tuple(q.shape)}")
            r.q_out_row_stride, r.q_out_head_stride = self._heads_of(q_out, "q_out")
            r.q_heads, r.d_q, r.d_q_out = q.shape[1], q.data_ptr(), q_out.data_ptr()
        self._run_rows(self._store, r, stream)
        return q_out

    def read(self, row_offset, length, *, rows, k=None, v=None, stream=None):
        """The last slots of sequences as rows: (k, v), each [rows, kv_heads, head_dim] of the cache's type.

        row_offset  [seqs + 1] int32: sequence s gives rows row_offset[s] .. row_offset[s + 1], its last slots of
        length      [seqs] int32; a length of as many rows is the sequence's beginning
        rows        of the tensors, >= row_offset[seqs]; those behind the last sequence are left as they are
        k, v        take the rows (default: new tensors)
        """
        r = _Rows()
        with self._on(stream):
            if k is None:
                k = self._torch.empty(rows, self.kv_heads, self.head_dim, dtype=self.dtype, device=self.device)
            if v is None:
                v = self._torch.empty(rows, self.kv_heads, self.head_dim, dtype=self.dtype, device=self.device)
        r.k_row_stride, r.k_head_stride = self._heads_of(k, "k", rows)
        r.v_row_stride, r.v_head_stride = self._heads_of(v, "v", rows)
        r.n_rows, r.max_len, r.d_k, r.d_v = rows, self.max_len, k.data_ptr(), v.data_ptr()
        r.d_row_offset, r.d_length = self._ints(row_offset, "row_offset", self.n_seqs + 1), self._ints(length, "length", self.n_seqs)
        self._run_rows(self._read, r, stream)
        return k, v
