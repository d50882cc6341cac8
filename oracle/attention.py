"""Float64 reference of the language side's attention: packed prompts and the 8-bit cache.

Plain numpy from the definitions (include/eas_attention.h); shares no code with the HIP library.
"""
import numpy as np


def attention(q, k, v, scale, sees):
    """One head: q [queries, dim], k, v [keys, dim]; query i sees the keys whose entry of sees [queries, keys] is
    true.  Returns (out, lse); a query that sees none gets zeros and -inf."""
    out = np.zeros((q.shape[0], v.shape[1]))
    lse = np.full(q.shape[0], -np.inf)
    for i in range(q.shape[0]):
        at = np.flatnonzero(sees[i])
        if at.size:
            s = scale * (k[at] @ q[i])
            top = s.max()
            e = np.exp(s - top)
            out[i] = e @ v[at] / e.sum()
            lse[i] = top + np.log(e.sum())
    return out, lse


def visible(lq, lk, causal):
    """[lq, lk]: the queries are the last lq of the lk tokens where causal."""
    i, j = np.arange(lq)[:, None], np.arange(lk)[None, :]
    return j <= i + lk - lq if causal else np.ones((lq, lk), bool)


def prompt_attention(q, k, v, cu_q, cu_k, scale, causal):
    """q [rows, heads, dim], k, v [rows, kv_heads, dim]; NaN in rows of no sequence."""
    group = q.shape[1] // k.shape[1]
    out, lse = np.full(q.shape, np.nan), np.full(q.shape[:2], np.nan)
    for r in range(len(cu_q) - 1):
        a, b = slice(cu_q[r], cu_q[r + 1]), slice(cu_k[r], cu_k[r + 1])
        sees = visible(a.stop - a.start, b.stop - b.start, causal)
        for h in range(q.shape[1]):
            out[a, h], lse[a, h] = attention(q[a, h], k[b, h // group], v[b, h // group], scale, sees)
    return out, lse


# ---- 8-bit codes ---------------------------------------------------------------

MOST = {"int8": 127.0, "e4m3": 448.0}
# the value of each non-negative e4m3 code: sign 1, exponent 4 (bias 7), mantissa 3; 0x7f is no number
E4M3 = np.array([(m / 8.0) * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7)
                 for e in range(16) for m in range(8)][:127])


def scale_of(top, most):
    """2^e with the smallest e >= -126 and top <= most * 2^e; 0 for top = 0."""
    if top == 0:
        return 0.0
    e = -126
    while top > most * 2.0 ** e:
        e += 1
    return 2.0 ** e


def encode(x, scale, form):
    """Codes as the values that they stand for, without the scale."""
    with np.errstate(invalid="ignore"):
        y = x / scale if scale else np.where(np.isinf(x), 0.0, x * 0.0)
    y = np.clip(np.where(np.isnan(y), 0.0, y), -MOST[form], MOST[form])
    if form == "int8":
        return np.rint(y)
    a = np.abs(y)
    hi = np.searchsorted(E4M3, a)                  # E4M3[hi - 1] < a <= E4M3[hi]
    lo = np.maximum(hi - 1, 0)
    up, down = E4M3[hi] - a, a - E4M3[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    return np.copysign(E4M3[code], y)


class Cache:
    """Blocks as values without scale, and scales."""

    def __init__(self, n_pages, kv_heads, page, dim, form):
        self.page, self.form = page, form
        self.code = {n: np.zeros((n_pages, kv_heads, page, dim)) for n in "kv"}
        self.scale = {n: np.zeros((n_pages, kv_heads)) for n in "kv"}

    def append(self, k, v, held, table):
        """One sequence: k, v [tokens, kv_heads, dim] behind `held` tokens, page by page."""
        n_pages = self.scale["k"].shape[0]
        for slot in range(held // self.page, len(table)):
            lo, hi = max(held, slot * self.page), min(held + k.shape[0], (slot + 1) * self.page)
            page = table[slot]
            if lo >= hi or not 0 <= page < n_pages:
                continue
            a, b = lo - slot * self.page, hi - slot * self.page
            for name, x in (("k", k), ("v", v)):
                for h in range(x.shape[1]):
                    new = x[lo - held:hi - held, h]
                    fin = np.abs(new[np.isfinite(new)])
                    s = scale_of(fin.max() if fin.size else 0.0, MOST[self.form])
                    if a > 0:
                        old = self.scale[name][page, h]
                        s = max(s, old)
                        if s > old:
                            self.code[name][page, h, :a] = encode(self.code[name][page, h, :a] * old, s, self.form)
                    self.scale[name][page, h] = s
                    self.code[name][page, h, a:b] = encode(new, s, self.form)

    def rows(self, name, table, first, n):
        """Tokens first .. first + n of a sequence [n, kv_heads, dim]; zeros where no page is held."""
        code, scale = self.code[name], self.scale[name]
        out = np.zeros((n, code.shape[1], code.shape[3]))
        for i in range(n):
            t = first + i
            if 0 <= t < len(table) * self.page and 0 <= table[t // self.page] < code.shape[0]:
                p = table[t // self.page]
                out[i] = code[p, :, t % self.page] * scale[p][:, None]
        return out

    def attention(self, q, length, table, scale, causal):
        """One sequence's queries [queries, heads, dim] over its first `length` tokens."""
        k, v = self.rows("k", table, 0, length), self.rows("v", table, 0, length)
        there = np.array([0 <= table[t // self.page] < self.scale["k"].shape[0] for t in range(length)], bool)
        sees = visible(q.shape[0], length, causal) & there[None, :]
        out, lse = np.zeros(q.shape), np.zeros(q.shape[:2])
        group = q.shape[1] // k.shape[1]
        for h in range(q.shape[1]):
            out[:, h], lse[:, h] = attention(q[:, h], k[:, h // group], v[:, h // group], scale, sees)
        return out, lse
