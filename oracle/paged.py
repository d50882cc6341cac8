"""Float64 reference of prompts in pieces: rotary positions with several axes and the paged 16-bit cache.

Plain numpy from the definitions (include/eas_paged.h); shares no code with the HIP library.
"""
import numpy as np

from . import attention as O


def angles(positions, freqs, axis):
    """[rows, pairs], reduced to one turn in numpy's longest float.  positions [axes, rows]."""
    p = np.asarray(positions, np.int64).astype(np.longdouble)[np.asarray(axis)].T
    a = p * np.asarray(freqs, np.float64).astype(np.longdouble)
    turn = 2 * np.longdouble(np.pi) + 2 * np.longdouble("1.22464679914735317722606593227500105e-16")   # pi and its rest
    return (a - np.round(a / turn) * turn).astype(np.float64)


def rotate(x, positions, freqs, axis, adjacent=False, inverse=False):
    """x [rows, heads, dim], each pair a complex number times e^(i angle)."""
    n = len(freqs)
    first = np.arange(n) * 2 if adjacent else np.arange(n)
    second = first + 1 if adjacent else first + n
    turn = np.exp((-1j if inverse else 1j) * angles(positions, freqs, axis))[:, None]
    z = (x[..., first] + 1j * x[..., second]) * turn
    out = np.array(x, np.float64)
    out[..., first], out[..., second] = z.real, z.imag
    return out


class Cache:
    """Pages [n_pages, heads, page, dim] of keys and values, filled with `fill`."""

    def __init__(self, n_pages, heads, page, dim, fill):
        self.k = np.full((n_pages, heads, page, dim), fill, np.float64)
        self.v = self.k.copy()
        self.page = page

    def append(self, k, v, held, table):
        """New tokens behind `held` of a sequence with pages `table`; those without a page are dropped."""
        for i in range(k.shape[0]):
            at, slot = divmod(held + i, self.page)
            if at < len(table) and 0 <= table[at] < self.k.shape[0]:
                self.k[table[at], :, slot], self.v[table[at], :, slot] = k[i], v[i]

    def attention(self, q, length, table, scale, causal):
        """q [queries, heads, dim] over the first `length` tokens of a sequence whose last Lq they are.  Tokens of pages
        that are not held are not seen.  Returns (out, lse, A = sum p |v|)."""
        lq, heads, dim = q.shape
        there = [t for t in range(length) if t // self.page < len(table) and 0 <= table[t // self.page] < self.k.shape[0]]
        k = np.stack([self.k[table[t // self.page], :, t % self.page] for t in there]) if there else \
            np.zeros((0,) + self.k.shape[1::2])
        v = np.stack([self.v[table[t // self.page], :, t % self.page] for t in there]) if there else k
        sees = O.visible(lq, length, causal)[:, there]
        group = heads // self.k.shape[1]
        out, lse, size = np.zeros(q.shape), np.zeros(q.shape[:2]), np.zeros(q.shape)
        for h in range(heads):
            kk, vv = k[:, h // group], v[:, h // group]
            out[:, h], lse[:, h] = O.attention(q[:, h], kk, vv, scale, sees)
            size[:, h], _ = O.attention(q[:, h], kk, np.abs(vv), scale, sees)
        return out, lse, size
