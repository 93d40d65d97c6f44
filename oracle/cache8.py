"""Keys and values in pages of 64 tokens as e4m3 with one power-of-two scale per page, head and K or V, and attention
over them, plain float64 NumPy (oracle: test infrastructure only).

* append: a tile's exponent is the smallest e in [-126, 127] that keeps its new finite values within 448 * 2^e, and not
  below what it was if the tile holds older tokens; those are then rounded anew, from the values that they stood for;
* a table entry that names no page: nothing is written, and its tokens are not there for the attention;
* attention: softmax over the tokens that a query sees; none: zeros.
"""
from __future__ import annotations

import math

import numpy as np

from . import fp8

PAGE = 64


def slot(t):
    """Where a tile of V holds token t of its page."""
    return 16 * (t // 4 % 4) + 4 * (t // 16) + t % 4


SLOTS = np.array([slot(t) for t in range(PAGE)])


class Cache:
    """Codes k [pages][heads][64][hd], v [pages][heads][hd][64] and scale bytes [pages][heads] as the library holds
    them; table [samples][pages of one]."""

    def __init__(self, k, v, k_scale, v_scale, table):
        self.k, self.v, self.ks, self.vs, self.table = k, v, k_scale, v_scale, np.asarray(table)

    @property
    def heads(self):
        return self.k.shape[1]

    def page(self, b: int, token: int) -> int:
        p = int(self.table[b, token // PAGE])
        return p if 0 <= p < self.k.shape[0] else -1

    def tile(self, is_v: bool, page: int, head: int) -> np.ndarray:
        """Codes [64 tokens][hd] of a tile (a copy)."""
        return self.v[page, head][:, SLOTS].T.copy() if is_v else self.k[page, head].copy()

    def put(self, is_v: bool, page: int, head: int, codes: np.ndarray):
        if is_v:
            self.v[page, head][:, SLOTS] = codes.T
        else:
            self.k[page, head] = codes

    def append(self, b: int, held: int, k: np.ndarray, v: np.ndarray):
        """Rows of k and v [n][heads * hd] become tokens held.. of sample b."""
        n, hd = k.shape[0], self.k.shape[3]
        at = 0
        while at < n:
            first = (held + at) % PAGE
            m = min(PAGE - first, n - at)
            page = self.page(b, held + at)
            for head in range(self.heads) if page >= 0 else ():
                for is_v, x, scale in ((False, k, self.ks), (True, v, self.vs)):
                    new = x[at:at + m, head * hd:(head + 1) * hd].astype(np.float64)
                    ok = np.isfinite(new)
                    e = fp8.block_exponent(float(np.abs(new[ok]).max()) if ok.any() else 0.0)
                    codes = self.tile(is_v, page, head)
                    if first:
                        was = int(scale[page, head]) - 127
                        e = max(e, was)
                        codes[:first] = fp8.encode(fp8.decode(codes[:first]) * math.ldexp(1.0, was - e))
                    codes[first:first + m] = fp8.encode(new * math.ldexp(1.0, -e))
                    self.put(is_v, page, head, codes)
                    scale[page, head] = e + 127
            at += m

    def rows(self, is_v: bool, b: int, n: int, head: int):
        """(values float64 [n][hd] of sample b's tokens, whether each is there)."""
        out = np.zeros((n, self.k.shape[3]))
        there = np.zeros(n, bool)
        for t in range(0, n, PAGE):
            page = self.page(b, t)
            if page >= 0:
                m = min(PAGE, n - t)
                e = int((self.vs if is_v else self.ks)[page, head]) - 127
                out[t:t + m] = fp8.decode(self.tile(is_v, page, head)[:m]) * math.ldexp(1.0, e)
                there[t:t + m] = True
        return out, there

    def attention(self, b: int, held: int, q: np.ndarray, causal: bool):
        """(outputs [n][H * hd], sums of p |v| [n][H * hd], largest sum of |q k| over a query's scores [n][H]) of
        queries q [n][H * hd]; p the softmax's probabilities."""
        n, hd = q.shape[0], self.k.shape[3]
        H = q.shape[1] // hd
        out, mag, top = np.zeros(q.shape), np.zeros(q.shape), np.zeros((n, H))
        for h in range(H):
            kv = h // (H // self.heads)
            (k, there), (v, _) = self.rows(False, b, held, kv), self.rows(True, b, held, kv)
            cols = slice(h * hd, (h + 1) * hd)
            for i in range(n):
                see = there.copy()
                if causal:
                    see &= np.arange(held) <= held - n + i
                if not see.any():
                    continue
                ks, vs = k[see], v[see]
                s = (ks @ q[i, cols].astype(np.float64)) / math.sqrt(hd)
                p = np.exp(s - s.max())
                p /= p.sum()
                out[i, cols], mag[i, cols] = p @ vs, p @ np.abs(vs)
                top[i, h] = (np.abs(ks) @ np.abs(q[i, cols].astype(np.float64))).max() / math.sqrt(hd)
        return out, mag, top
