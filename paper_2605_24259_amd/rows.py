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


def share(a, b):
    """Whether rows a and b, [rows, heads, dim] with the last dimension contiguous, may share elements: found wherever they do,
    and not where they lie one behind the other, side by side in the rows of one tensor, or head between heads."""
    if a.untyped_storage().data_ptr() != b.untyped_storage().data_ptr() or not a.numel() or not b.numel():
        return False
    (rows, heads, dim), at = a.shape, (b.data_ptr() - a.data_ptr()) // a.element_size()
    (row, head, _), (row_b, head_b, _) = a.stride(), b.stride()
    in_row, in_row_b = (heads - 1) * head + dim, (b.shape[1] - 1) * head_b + b.shape[2]
    if at >= (rows - 1) * row + in_row or -at >= (b.shape[0] - 1) * row_b + in_row_b:
        return False
    if rows > 1 and row != row_b or b.shape != a.shape or heads > 1 and head != head_b:
        return True
    if rows > 1 and row and in_row <= at % row <= row - in_row_b:
        return False
    for n, stride in sorted(((rows, row), (heads, head), (2, abs(at))), key=lambda x: x[1]):  # from the nearest on
        if n > 1 and stride < dim:
            return True
        dim += (n - 1) * stride
    return False


def moves(a, b):
    """Whether writing what comes of rows a into rows b, of the same shape, may change other rows or heads of a."""
    if a is b or a.data_ptr() == b.data_ptr() and all(n == 1 or x == y for n, x, y in zip(a.shape, a.stride(), b.stride())):
        return False
    return share(a, b)


class RowOps:
    """``store`` and ``read`` of a cache with the fields of ``PagedCache``; ``_store`` and ``_read`` are the library's
    functions."""

    def _heads_of(self, t, name, shape):
        """Strides of a tensor of rows, of a dimension of one 0, as they say nothing."""
        at, heads, last = t.stride() if t.dim() == 3 else (0, 0, 0)
        if last != 1 or t.shape != shape or t.dtype is not self.dtype or t.get_device() != self._index:
            raise ValueError(f"{name}: {tuple(shape)} of {self.dtype} on {self.device}, the last dimension contiguous, is wanted, got "
                             f"{t.dtype} {tuple(t.shape)} on {t.device}")
        return at if shape[0] > 1 else 0, heads if shape[1] > 1 else 0

    def _new_rows(self, shape):
        return self._torch.empty_strided(shape, (self.kv_heads * self.head_dim, self.head_dim, 1), dtype=self.dtype, device=self.device)

    def _norm_of(self, t, name, kind):
        if t.dtype is not kind or (kind is not self.dtype and kind is not self._torch.float32) or t.get_device() != self._index or \
                t.shape != (self.head_dim,) or not t.is_contiguous():
            raise ValueError(f"{name}: a contiguous tensor [{self.head_dim}] of {self.dtype} or float32 (both norms alike) on "
                             f"{self.device} is wanted, got {t.dtype} {tuple(t.shape)} on {t.device}")
        return t.data_ptr()

    def _run_rows(self, f, args, stream):
        st = f(self._c_ref, ctypes.byref(_Rows(*args)), self._raw_stream(self._index) if stream is None else _stream_ptr(stream))
        if st != 0:
            raise RkcError(st, f.__name__)

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
        q_out       takes the queries; may be q, and shares no other memory with q, k or v

        Returns the queries (q_out or a new tensor), or None without q.  A cache of 4 bits rounds keys and values as they
        are written; keys are computed in 64 bits up to that.
        """
        torch = self._torch
        shape = (k.shape[0] if k.dim() else 0, self.kv_heads, self.head_dim)
        n = shape[0]
        k_at, k_heads = self._heads_of(k, "k", shape)
        v_at, v_heads = self._heads_of(v, "v", shape)
        offsets, lengths = self._ints(row_offset, "row_offset", self.n_seqs + 1), self._ints(length, "length", self.n_seqs)
        f32, qn, kn = False, None, None
        if q_norm is not None or k_norm is not None:
            kind = (k_norm if q_norm is None else q_norm).dtype
            f32 = kind is torch.float32
            if q_norm is not None:
                qn = self._norm_of(q_norm, "q_norm", kind)
            if k_norm is not None:
                kn = self._norm_of(k_norm, "k_norm", kind)
        pairs, freqs, axes, positions, axis_of = 0, None, 1, None, None
        if freq is not None:
            pairs = freq.shape[0] if freq.dim() == 1 else -1
            if freq.dtype is not torch.float32 or freq.get_device() != self._index or pairs % 8 or not 0 <= 2 * pairs <= self.head_dim or \
                    not freq.is_contiguous():
                raise ValueError(f"freq: a contiguous float32 tensor of 8, 16, ... {self.head_dim // 2} values on {self.device} is wanted, "
                                 f"got {freq.dtype} {tuple(freq.shape)} on {freq.device}")
            freqs = freq.data_ptr()
        if position is not None:
            of = position.shape
            if len(of) == 2:
                axes = of[0]
            if position.dtype is not torch.int32 or position.get_device() != self._index or len(of) not in (1, 2) or of[-1] != n or \
                    not 1 <= axes <= MAX_AXES or not position.is_contiguous():
                raise ValueError(f"position: a contiguous int32 tensor [{n}] or [up to {MAX_AXES}, {n}] on {self.device} is wanted, got "
                                 f"{position.dtype} {tuple(of)} on {position.device}")
            positions = position.data_ptr()
        if axis is not None:
            if position is None or freq is None:
                raise ValueError("axis: there are several axes only of given positions and frequencies")
            axis_of = self._ints(axis, "axis", pairs)
        elif axes > 1 and pairs:
            raise ValueError(f"position: of {axes} axes, axis has to say which one each of the {pairs} pairs turns by")
        elif axes > 1:
            axes, positions = 1, None  # nothing turns
        heads, queries, outs, q_at, q_heads, out_at, out_heads = 0, None, None, 0, 0, 0, 0
        if q is not None:
            heads = q.shape[1] if q.dim() == 3 else 0
            shape = (n, heads, self.head_dim)
            q_at, q_heads = self._heads_of(q, "q", shape)
            if q_out is None:
                if stream is None:  # a context, even an empty one, costs a fifth of a tensor
                    q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
                else:
                    with self._on(stream):
                        q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
                out_at, out_heads = heads * self.head_dim, self.head_dim
            else:
                out_at, out_heads = self._heads_of(q_out, "q_out", shape)
                if moves(q, q_out):
                    raise RkcError(-3, f"{self._store.__name__}: q_out may be q, but not share elements with other rows or heads of it")
            queries, outs = q.data_ptr(), q_out.data_ptr()
        elif q_norm is not None or q_out is not None:
            raise ValueError("q_norm and q_out are of queries, and there are none")
        self._run_rows(self._store, (n, heads, self.max_len, pairs, axes, interleaved, f32, eps, k_at, k_heads, v_at, v_heads, q_at, q_heads,
                                     out_at, out_heads, k.data_ptr(), v.data_ptr(), queries, outs, offsets, lengths, positions, axis_of,
                                     freqs, qn, kn), stream)
        return q_out

    def read(self, row_offset, length, *, rows, k=None, v=None, stream=None):
        """The last slots of sequences as rows: (k, v), each [rows, kv_heads, head_dim] of the cache's type.

        row_offset  [seqs + 1] int32: sequence s gives rows row_offset[s] .. row_offset[s + 1], its last slots of
        length      [seqs] int32; a length of as many rows is the sequence's beginning
        rows        of the tensors, >= row_offset[seqs]; those behind the last sequence are left as they are
        k, v        take the rows (default: new tensors)
        """
        shape, torch = (rows, self.kv_heads, self.head_dim), self._torch
        given = k is not None and v is not None
        if not given:
            if stream is not None:
                with self._on(stream):
                    k, v = self._new_rows(shape) if k is None else k, self._new_rows(shape) if v is None else v
            else:
                k, v = self._new_rows(shape) if k is None else k, self._new_rows(shape) if v is None else v
        k_at, k_heads = self._heads_of(k, "k", shape)
        v_at, v_heads = self._heads_of(v, "v", shape)
        if given and share(k, v):
            raise RkcError(-3, f"{self._read.__name__}: k and v share elements")
        self._run_rows(self._read, (rows, 0, self.max_len, 0, 1, 0, 0, 0.0, k_at, k_heads, v_at, v_heads, 0, 0, 0, 0, k.data_ptr(), v.data_ptr(),
                                    None, None, self._ints(row_offset, "row_offset", self.n_seqs + 1), self._ints(length, "length", self.n_seqs)),
                       stream)
        return k, v
