"""Plain implementation of rows into a paged cache (norm, rotation, 4 bits) and back, in 64 bits on the CPU."""
from __future__ import annotations

import numpy as np

from tests import cache_reference as ref

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
TOP = {"bfloat16": 125, "float16": 13}  # exponent of the largest scale


def held(x, dtype):
    """(codes, scale bytes, values) of finite x [..., D], 32 bits."""
    x = np.asarray(x, np.float32).astype(np.float64)
    b = x.reshape(x.shape[:-1] + (-1, 32))
    most = np.abs(b).max(-1)
    m, e = np.frexp(most)  # most = m 2^e, m in [1/2, 1)
    e = np.clip(np.where(m <= 7 / 8, e - 3, e - 2), -126, TOP[dtype])
    e = np.where(most == 0, -126, e)
    y = np.abs(b) / 2.0 ** e[..., None]
    off = np.abs(y[..., None] - VALUES)
    # the nearest, of two as near the even one
    best = off.min(-1, keepdims=True)
    code = np.where((off == best) & (np.arange(8) % 2 == 0), 8 - np.arange(8), np.where(off == best, 0.5, 0)).argmax(-1)
    value = np.copysign(VALUES[code], b) * 2.0 ** e[..., None]
    code = code + 8 * np.signbit(b)
    return code.reshape(x.shape).astype(np.uint8), (e + 127).astype(np.uint8), value.reshape(x.shape)


def values(code, scale):
    """[..., D] codes and [..., D / 32] bytes."""
    x = VALUES[code & 7] * np.where(code & 8, -1.0, 1.0)
    return (x.reshape(x.shape[:-1] + (-1, 32)) * 2.0 ** (scale.astype(np.float64)[..., None] - 127)).reshape(x.shape)


def split(pool, page, dim):
    """Keys' codes, values' codes, keys' and values' scale bytes of a pool [blocks, heads, bytes]: [blocks, heads, page, ...]."""
    n, m = page * dim // 2, page * dim // 32
    c = pool[..., :2 * n].reshape(pool.shape[:2] + (2, page, dim // 2))
    c = np.stack([c & 15, c >> 4], -1).reshape(pool.shape[:2] + (2, page, dim))
    s = pool[..., 2 * n:].reshape(pool.shape[:2] + (2, page, dim // 32))
    return c[:, :, 0], c[:, :, 1], s[:, :, 0], s[:, :, 1]


def joined(kc, vc, ks, vs):
    """The pool of them."""
    def codes(c):
        return (c[..., 0::2] | c[..., 1::2] << 4).reshape(c.shape[:2] + (-1,))
    return np.concatenate([codes(kc), codes(vc), ks.reshape(ks.shape[:2] + (-1,)), vs.reshape(vs.shape[:2] + (-1,))], -1).astype(np.uint8)


def turned(x, weight, eps, freq, position, axis, interleaved):
    """Norm and rotation of x [rows, heads, D]; position [axes, rows]."""
    x = np.asarray(x, np.float64)
    with np.errstate(all="ignore"):
        if weight is not None:
            x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
        if freq is None:
            return x
        y, n = x.copy(), len(freq)
        for j in range(n):
            # the angle in turns, exactly up to the last step
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + n)
            t = [whole_angle(int(p), float(freq[j])) for p in position[0 if axis is None else axis[j]]]
            c, s = np.cos(t)[:, None], np.sin(t)[:, None]
            y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


_PI = 3141592653589793238462643383279502884197169399375105820974944592307816406286  # 10^75 pi


def whole_angle(position, freq):
    """position * freq less whole turns, with whole numbers."""
    from fractions import Fraction
    x = Fraction(position) * Fraction(freq)
    turn = Fraction(2 * _PI, 10 ** 75)
    return float(x - turn * round(x / turn))


class Packed(ref.Case):
    """The sequences and rows of a Case over a cache of 4 bits: k and v become the values held, the pool is `pool`."""

    def __init__(self, *a, marks=(), **kw):
        super().__init__(*a, **kw)
        import torch
        name = str(self.dtype).split(".")[1]
        k, v = (np.nan_to_num(x.double().numpy(), nan=0, posinf=0, neginf=0).transpose(0, 2, 1, 3) for x in (self.k, self.v))
        (kc, ks, kv), (vc, vs, vv) = held(k, name), held(v, name)
        kv, vv = kv.copy(), vv.copy()
        for s, j, h in marks:  # heads of slots that are not numbers
            b, i = int(self.table[s, j // self.page]), j % self.page
            ks[b, h, i, 0] = 255
            kv[b, h, i] = vv[b, h, i] = np.nan
        # behind the lengths and in blocks of nobody: bytes of ones
        mine = np.zeros(k.shape[:3], bool)
        for s, n in enumerate(self.lens):
            for j in range(n):
                mine[int(self.table[s, j // self.page]), :, j % self.page] = True
        for x in (kc, vc, ks, vs):
            x[~mine] = 255 if x is ks or x is vs else 15
        self.pool = torch.from_numpy(joined(kc, vc, ks, vs))
        self.k, self.v = (torch.from_numpy(x.transpose(0, 2, 1, 3).copy()) for x in (kv, vv))


    def attend_at_once(self):
        """``attend`` for finite values, a head's rows at once."""
        T, Q = self.q.shape[:2]
        out, lse = np.zeros((T, Q, self.dim)), np.full((T, Q), -np.inf)
        for s in range(len(self.lens)):
            rows = slice(int(self.offset[s]), int(self.offset[s + 1]))
            for h in range(self.kv_heads):
                v = self.slots(self.v, s, h)
                for head in range(h * self.group, (h + 1) * self.group):
                    x, see = self.scores(s, head)
                    x = np.where(see, x, -np.inf)
                    m = x.max(-1, initial=-np.inf, keepdims=True)
                    p = np.exp(x - np.where(m == -np.inf, 0, m))
                    total = p.sum(-1, keepdims=True)
                    with np.errstate(divide="ignore"):
                        lse[rows, head] = (m + np.log(total))[:, 0]
                    out[rows, head] = p @ v / np.where(total == 0, 1, total)
        return out, lse

    def slots(self, pool, s, h):
        n, j = self.lens[s], np.arange(self.lens[s])
        return pool[self.table[s].numpy()[j // self.page], j % self.page, h].double().numpy() if n else np.zeros((0, self.dim))
