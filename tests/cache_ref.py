"""The cache of 8-bit pages and its attention as their formulas say, in NumPy: scales in 32 bits as they are held, the rest in 64."""
import math

import numpy as np

PAGE = 64
F = np.float32


class RefCache:
    """codes[page] = [heads, 64, dim] integers, scale[page] = [heads]; one of keys or values."""

    def __init__(self, pages, heads, dim):
        self.codes = np.zeros((pages, heads, PAGE, dim), np.int64)
        self.scale = np.zeros((pages, heads), F)

    def store(self, x, table, starts, held):
        """x [tokens, heads, dim] float64 (values of the storage type)."""
        pages = self.scale.shape[0]
        for s in range(len(held)):
            rows, at = x[starts[s]:starts[s + 1]], held[s]
            while len(rows):
                slot, off = at // PAGE, at % PAGE
                n = min(PAGE - off, len(rows))
                page = table[s][slot] if slot < len(table[s]) else -1
                if 0 <= page < pages:
                    self._page(page, off, rows[:n])
                rows, at = rows[n:], at + n

    def _page(self, page, off, x):
        for h in range(self.scale.shape[1]):
            v = x[:, h]
            top = np.abs(v).max() if np.isfinite(v).all() else np.nan
            need, old = F(F(top) / F(127)), self.scale[page, h]
            new = need
            if off:
                if need <= old:
                    new = old
                else:
                    new = F(np.nan) if np.isnan(need) or np.isnan(old) else max(need, F(F(1.25) * old))
                    ratio = F(old / new) if new > 0 else F(0)
                    self.codes[page, h, :off] = np.rint(self.codes[page, h, :off].astype(F) * ratio)
            self.scale[page, h] = new
            # the quotient rounded to 32 bits, then to a whole number: both as IEEE says
            self.codes[page, h, off:off + len(v)] = np.clip(np.rint(v.astype(F) / new), -127, 127) if new > 0 else 0

    def values(self, table_row, n):
        """[n, heads, dim] float64 of the first n tokens, and which of them have a page."""
        out, there = np.zeros((n, self.scale.shape[1], self.codes.shape[3])), np.zeros(n, bool)
        for i in range(-(-n // PAGE)):
            page = table_row[i] if i < len(table_row) else -1
            if 0 <= page < self.scale.shape[0]:
                m = min(PAGE, n - i * PAGE)
                out[i * PAGE:i * PAGE + m] = (self.codes[page, :, :m] * self.scale[page].astype(np.float64)[:, None, None]).transpose(1, 0, 2)
                there[i * PAGE:i * PAGE + m] = True
        return out, there


def attend(q, k, v, there, causal, window, mask, scale):
    """One sequence: q [n, heads, dim], k, v [L, kv_heads, dim] float64 -> out, log-sum."""
    n, heads, dim = q.shape
    L, g = len(k), heads // k.shape[1]
    out, lse = np.zeros((n, heads, dim)), np.full((n, heads), -np.inf)
    for i in range(n):
        sees = there.copy()
        if causal:
            at = L - n + i
            sees &= np.arange(L) <= at
            if window:
                sees &= np.arange(L) > at - window
        if mask is not None:
            sees &= mask[:L] != 0
        if not sees.any():
            continue
        for h in range(heads):
            s = scale * (k[sees, h // g] @ q[i, h])
            top = s.max()
            p = np.exp(s - top)
            out[i, h] = p @ v[sees, h // g] / p.sum()
            lse[i, h] = top + math.log(p.sum())
    return out, lse
