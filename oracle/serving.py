"""Plain 64-bit forms of the operators of low-bit language models (numpy): 8-bit codes with a scale for each row, their
scaled products, the paged 4-bit cache and the attention that reads it.  Inputs are float64 arrays that hold the values of
whatever 16- or 32-bit type the operator is given."""

from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
LOWEST, HIGHEST = -23, 13           # exponents of the 4-bit groups' powers of two


def quantize_tokens(x):
    """[rows, K] -> codes (int8 [rows, K rounded up to 16]) and scales (fp32 [rows])."""
    x = np.asarray(x, np.float64)
    rows, K = x.shape
    codes, scale = np.zeros((rows, -(-K // 16) * 16), np.int8), np.zeros(rows, np.float32)
    for r in range(rows):
        if not np.isfinite(x[r]).all():
            scale[r] = np.nan
            continue
        top = np.abs(x[r]).max(initial=0.0)
        scale[r] = np.float32(top) / np.float32(127)
        if top > 0:
            codes[r, :K] = np.rint(127 * x[r] / top)    # the quotient of two numbers of 31 and 24 bits: a tie is one in 64 bits, and only a tie is
    return codes, scale


def gemm_scaled(X, x_scale, W, w_scale, bias=None):
    """float64 [M, N], the integer sums exact."""
    total = X.astype(np.float64) @ W.astype(np.float64).T
    y = total * x_scale.astype(np.float64)[:, None] * w_scale.astype(np.float64)
    return y if bias is None else y + bias.astype(np.float64)


def encode4(x):
    """[..., D] -> codes (0 .. 15, [..., D]) and exponents ([..., D / 32])."""
    g = np.asarray(x, np.float64).reshape(*np.shape(x)[:-1], -1, 32)
    top = np.abs(g).max(-1)
    e = np.full(top.shape, HIGHEST)
    for x_ in range(HIGHEST - 1, LOWEST - 1, -1):
        e = np.where(top < 7 * 2.0 ** x_, x_, e)
    u = np.minimum(np.abs(g) / 2.0 ** e[..., None], 6)  # beyond the largest: that one
    distance = np.abs(u[..., None] - MAGNITUDES)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])          # of two equally near the even code
    code = order[np.argmin(distance[..., order], -1)]
    return (code + 8 * (np.signbit(g))).reshape(np.shape(x)).astype(np.uint8), e


def decode4(code, e):
    """Values of codes ([..., D]) with exponents ([..., D / 32])."""
    return np.where(code & 8, -1.0, 1.0) * MAGNITUDES[code & 7] * np.repeat(2.0 ** np.asarray(e, np.float64), 32, -1)


def rotate(x, table, positions, interleaved):
    """[tokens, heads, D], fp32 values of the rotation computed in 64 bits."""
    rot = table.shape[1]
    y = np.array(x, np.float64)
    cos, sin = (table[positions].astype(np.float64)[:, None, s] for s in (slice(0, rot // 2), slice(rot // 2, rot)))
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = y[..., first].copy(), y[..., second].copy()
    y[..., first], y[..., second] = a * cos - b * sin, b * cos + a * sin
    return y.astype(np.float32).astype(np.float64)


class Cache:
    """Values (float64, NaN for a (token, head) held as NaN) of every slot: [slots, heads, D]."""

    def __init__(self, pages, heads, page_size, D):
        self.pages, self.heads, self.page_size, self.D = pages, heads, page_size, D
        self.k = np.zeros((pages * page_size, heads, D))
        self.v = np.zeros((pages * page_size, heads, D))

    def append(self, k, v, slots):
        """k already rotated."""
        for t, s in enumerate(slots):
            if 0 <= s < len(self.k):
                for h in range(self.heads):
                    if np.isfinite(k[t, h]).all() and np.isfinite(v[t, h]).all():
                        self.k[s, h], self.v[s, h] = decode4(*encode4(k[t, h])), decode4(*encode4(v[t, h]))
                    else:
                        self.k[s, h] = self.v[s, h] = np.nan


def attention(q, k, v, first, scale):
    """One head: queries [n, D] of which number i sees tokens 0 .. first + i of k, v [l, D] -> result, and
    sum p |v| and the largest sum |q k| scale a row has, from which a bound on the error follows."""
    n, l = len(q), len(k)
    out, spread, reach = np.zeros((n, q.shape[1])), np.zeros((n, q.shape[1])), np.zeros(n)
    for i in range(n):
        seen = min(max(first + i + 1, 0), l)
        if seen == 0:
            continue
        s = scale * (k[:seen] @ q[i])
        p = np.exp(s - s.max())
        p /= p.sum()
        out[i], spread[i] = p @ v[:seen], p @ np.abs(v[:seen])
        reach[i] = abs(scale) * (np.abs(k[:seen]) @ np.abs(q[i])).max()
    return out, spread, reach
