"""The 4-bit key/value cache and attention over it, plainly: the page layout of
include/eq.h written out byte by byte, the rounding to codes, and attention in
64 bits with a bound for what the kernels may be off."""
import math

import numpy as np

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)


def page_bytes(kv_heads, dim, page):
    return head_bytes(dim, page) * kv_heads


def head_bytes(dim, page):
    return -(-(page * dim + page * dim // 32 + page) // 128) * 128


def to_codes(x):
    """(codes, scale byte) of one group of fp32 values."""
    x = np.asarray(x, dtype=np.float32)
    if not np.isfinite(x).all():
        return None, 255
    top = float(np.abs(x).max())
    e = -103
    if top > 0:
        m, k = math.frexp(top)          # top = 2m 2^(k-1), 1 <= 2m < 2
        e = min(max(k - 1 - 2 + (2 * m >= 1.75), -103), 125)
    y = np.abs(x.astype(np.float64)) * 2.0 ** -e
    d = np.abs(y[:, None] - VALUES[None, :])
    near = np.argmin(d, axis=1)         # the lower neighbour on a tie
    up = np.minimum(near + 1, 7)
    tie = (d[np.arange(len(y)), near] == d[np.arange(len(y)), up]) & (up != near)
    codes = np.where(tie & (near % 2 == 1), up, near)
    return (codes | (np.signbit(x).astype(np.int64) << 3)).astype(np.uint8), e + 127


def from_codes(codes, byte):
    v = VALUES[codes & 7] * 2.0 ** (int(byte) - 127)
    v = np.where(codes & 8, -v, v)
    return np.full(v.shape, np.nan) if byte == 255 else v


class Pool:
    """Pages as bytes on the host."""

    def __init__(self, n_pages, page, kv_heads, dim, fill=0):
        self.page, self.heads, self.dim = page, kv_heads, dim
        self.hb = head_bytes(dim, page)
        self.raw = np.full((n_pages, self.hb * kv_heads), fill, dtype=np.uint8)

    def _key_scale(self, head, t, g):
        return (head * self.hb + self.page * self.dim + t // 16 * (self.dim // 2) +
                (t % 4 * (self.dim // 32) + g) * 4 + t % 16 // 4)

    def _value_scale(self, head, t):
        return head * self.hb + self.page * self.dim + self.page * self.dim // 32 + t

    def _value_bytes(self, head, t):
        c = np.arange(self.dim)
        return head * self.hb + self.page * self.dim // 2 + (t // 32 * self.dim + c) * 16 + t % 32 // 2

    def put(self, page, t, head, k, v):
        """Token t of a page: k and v fp32 [dim].  A group that is not finite
        keeps whatever codes it had (they stand for nothing)."""
        row = self.raw[page]
        for g in range(self.dim // 32):
            c, b = to_codes(k[32 * g:32 * g + 32])
            row[self._key_scale(head, t, g)] = b
            if c is not None:
                at = head * self.hb + t * (self.dim // 2) + 16 * g
                row[at:at + 16] = c[0::2] | c[1::2] << 4
        c, b = to_codes(v)
        row[self._value_scale(head, t)] = b
        if c is not None:
            at = self._value_bytes(head, t)
            row[at] = (row[at] & 15) | c << 4 if t % 2 else (row[at] & 240) | c

    def get(self, page, t, head):
        """(keys, values) of token t in 64 bits."""
        row = self.raw[page]
        at = head * self.hb + t * (self.dim // 2)
        b = row[at:at + self.dim // 2]
        c = np.stack((b & 15, b >> 4), axis=1).reshape(-1)
        k = np.concatenate([from_codes(c[32 * g:32 * g + 32], row[self._key_scale(head, t, g)])
                            for g in range(self.dim // 32)])
        c = row[self._value_bytes(head, t)] >> (4 * (t % 2)) & 15
        return k, from_codes(c, row[self._value_scale(head, t)])


def rotate32(x, cos, sin, pairs):
    """x fp32 [..., D] rotated by fp32 rows [..., half], each product and sum rounded."""
    x = np.array(x, dtype=np.float32)
    half = cos.shape[-1]
    a = x[..., 0:2 * half:2].copy() if pairs else x[..., :half].copy()
    b = x[..., 1:2 * half:2].copy() if pairs else x[..., half:2 * half].copy()
    u, v = a * cos - b * sin, b * cos + a * sin
    assert u.dtype == np.float32
    if pairs:
        x[..., 0:2 * half:2], x[..., 1:2 * half:2] = u, v
    else:
        x[..., :half], x[..., half:2 * half] = u, v
    return x


def norm64(x, w, eps):
    x = np.asarray(x, dtype=np.float64)
    if w is None:
        return x
    return x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * np.asarray(w, dtype=np.float64)


def rotate64(x, cos, sin, pairs):
    x = np.array(x, dtype=np.float64)
    half = cos.shape[-1]
    i, j = ((slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if pairs else
            (slice(0, half), slice(half, 2 * half)))
    a, b, c, s = x[..., i].copy(), x[..., j].copy(), cos.astype(np.float64), sin.astype(np.float64)
    x[..., i], x[..., j] = a * c - b * s, b * c + a * s
    return x


def attention64(q, k, v, wt, scale, seen):
    """One head: q [n, D], k and v [T, D], wt [T] the value scales, seen [n, T]
    booleans; all in 64 bits.  Returns (out [n, D], how far off the kernel may be
    [n, D]); rows that see nothing are zeros.

    The bound.  Scores are sums of 128 exact products in fp32: off by at most
    2^-16 of the sum of their magnitudes, and exp2, the sum of P and the final
    scaling by 2^-18 relative; w P is held to 2^-8 of itself or 2^-21 of the
    column's largest, whichever is more; the result is rounded to BF16, 2^-8."""
    n = q.shape[0]
    out, bound = np.zeros((n, v.shape[1])), np.zeros((n, v.shape[1]))
    s = q @ k.T * scale
    mass = np.abs(q) @ np.abs(k).T * scale
    for i in range(n):
        at = seen[i]
        if not at.any():
            continue
        z = s[i, at]
        p = np.exp(z - z.max())
        y = p * wt[at]
        codes = np.abs(v[at]) / wt[at][:, None]
        out[i] = p @ v[at] / p.sum()
        soft = 2.0 ** -16 * mass[i, at].max() + 2.0 ** -18
        per = np.maximum(2.0 ** -8 * y, 2.0 ** -21 * y.max())
        bound[i] = ((per @ codes) + 2 * soft * (p @ np.abs(v[at]))) / p.sum() + \
            2.0 ** -8 * np.abs(out[i])
    return out, bound * 1.02 + 1e-30
