"""8-bit rows and the operators on them, plain float64 NumPy (oracle: test infrastructure only).

* e4m3 (OCP): sign, 4 exponent bits with bias 7, 3 mantissa bits, largest 448, no infinities, NaN = 0x7f / 0xff;
* E8M0: one byte, the power of two 2^(byte - 127);
* quantisation of a block: the smallest 2^e, e in [-126, 127], with |x| <= 448 * 2^e over its finite x; x / 2^e rounded
  to the nearest e4m3 value, ties to the even mantissa; NaN and infinities become NaN;
* products of quantised matrices, GELU (tanh form), and the pass between two blocks.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 128


def _code_values() -> np.ndarray:
    v = []
    for c in range(127):
        e, m = c >> 3, c & 7
        v.append(math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10))
    return np.array(v)


VALUES = _code_values()                # of the codes 0..126, ascending


def decode(codes: np.ndarray) -> np.ndarray:
    codes = np.asarray(codes, np.uint8)
    mag = np.append(VALUES, np.nan)[codes & 0x7F]
    return np.where(codes & 0x80, -mag, mag)


def encode(x: np.ndarray) -> np.ndarray:
    """Codes of the nearest e4m3 values (|x| <= 448, ties to even codes); NaN and infinities: 0x7f."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    assert np.all(a <= 448.0)
    hi = np.searchsorted(VALUES, a)                # first value >= a
    lo = np.maximum(hi - 1, 0)
    hi = np.minimum(hi, len(VALUES) - 1)
    dl, dh = a - VALUES[lo], VALUES[hi] - a
    c = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)
    c = c | np.where(np.signbit(x), 0x80, 0)
    return np.where(np.isfinite(x), c, 0x7F).astype(np.uint8)


def block_exponent(amax: float) -> int:
    """The smallest e in [-126, 127] with amax <= 448 * 2^e."""
    e = -126
    if amax > 0:
        m, x = math.frexp(amax)
        e = x - 9 if m <= 0.875 else x - 8
    return min(max(e, -126), 127)


def quantise(x: np.ndarray, block_rows: int = 1):
    """(codes [R][K] uint8, scale bytes [ceil(R / block_rows)][ceil(K / 128)] uint8)."""
    x = np.asarray(x, np.float64)
    R, K = x.shape
    rb, kb = -(-R // block_rows), -(-K // BLOCK)
    codes, scale = np.empty((R, K), np.uint8), np.empty((rb, kb), np.uint8)
    for i in range(rb):
        for j in range(kb):
            s = np.s_[i * block_rows:(i + 1) * block_rows, j * BLOCK:(j + 1) * BLOCK]
            a = np.abs(x[s])
            a = a[np.isfinite(a)]
            e = block_exponent(float(a.max()) if a.size else 0.0)
            codes[s] = encode(np.ldexp(x[s], -e))
            scale[i, j] = e + 127
    return codes, scale


def scales(scale: np.ndarray, rows: int, cols: int, block_rows: int = 1) -> np.ndarray:
    """The scale of each element."""
    s = np.ldexp(1.0, np.asarray(scale, np.int64) - 127)
    return np.repeat(np.repeat(s, block_rows, 0)[:rows], BLOCK, 1)[:, :cols]


def dequantise(codes: np.ndarray, scale: np.ndarray, block_rows: int = 1) -> np.ndarray:
    return decode(codes) * scales(scale, *codes.shape, block_rows)


def gelu(x: np.ndarray) -> np.ndarray:
    return 0.5 * x * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x ** 3)))


def linear(a: np.ndarray, w: np.ndarray, bias=None) -> np.ndarray:
    v = a @ w.T
    return v if bias is None else v + bias


def norm(x: np.ndarray, kind: str, eps: float) -> np.ndarray:
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(axis=1, keepdims=True)
    return x / np.sqrt((x * x).mean(axis=1, keepdims=True) + eps)


def resid_norm(h, y=None, off=None, post="none", pre="layer", post_w=None, pre_w=None, gate=None, resid_scale=1.0,
               shift=None, scale=None, eps=1e-6):
    """(h, u) of the pass between two blocks; gate, shift, scale [B][d]; rows outside the offsets keep h and get 0."""
    h = np.array(h, np.float64)
    u = np.zeros_like(h)
    off = [0, h.shape[0]] if off is None else off
    for b, (lo, hi) in enumerate(zip(off, off[1:])):
        if lo == hi:
            continue
        r = np.s_[lo:hi]
        if y is not None:
            p = norm(np.asarray(y[r], np.float64), post, eps)
            p = p if post_w is None else p * post_w
            p = p if gate is None else p * gate[b]
            h[r] = h[r] + resid_scale * p
        v = norm(h[r], pre, eps)
        v = v if pre_w is None else v * pre_w
        u[r] = v if scale is None else v * (1.0 + scale[b]) + shift[b]
    return h, u
