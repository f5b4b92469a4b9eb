"""The 8-bit cache in 64-bit NumPy, element by element from its definition (used by
the tests of the calls that write and read it)."""
from __future__ import annotations

import numpy as np

FORMATS = ("e4m3", "int8")

# the magnitudes of the e4m3 codes 0x00..0x7E (0x7F is NaN)
_C = np.arange(0x7F)
E4M3 = np.where(_C < 8, (_C & 7) * 2.0 ** -9, (8 + (_C & 7)) * 2.0 ** ((_C >> 3) - 10.0))


def decode_codes(codes: np.ndarray, fmt: str) -> np.ndarray:
    if fmt == "int8":
        return codes.view(np.int8).astype(np.float64)
    c = codes.view(np.uint8)
    mag = np.append(E4M3, np.nan)[c & 0x7F]
    return np.where(c & 0x80, -mag, mag)


def encode_values(y: np.ndarray, fmt: str) -> np.ndarray:
    """Codes (uint8) nearest to y, ties to the even code, beyond the largest to the largest."""
    if fmt == "int8":
        return np.clip(np.rint(y), -127, 127).astype(np.int8).view(np.uint8)
    a = np.minimum(np.abs(y), 448.0)
    hi = np.clip(np.searchsorted(E4M3, a), 0, 0x7E)          # first code with magnitude >= a
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - E4M3[lo], E4M3[hi] - a
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (c | np.where(np.signbit(y), 0x80, 0)).astype(np.uint8)


def scale_of(amax: float, fmt: str) -> float:
    if amax == 0:
        return 0.0
    if fmt == "e4m3":
        e = -126
        while amax > 448.0 * 2.0 ** e:
            e += 1
        return 2.0 ** e
    return float(max(np.float32(amax) / np.float32(127.0), np.float32(2.0 ** -126)))


def append(codes, scales, x, offset, block, fmt):
    """Rows x [m][D] (float64) into codes [cap][D] uint8 / scales [blocks] float64, in place."""
    m = len(x)
    if m == 0:
        return
    for blk in range(offset // block, (offset + m - 1) // block + 1):
        r0 = blk * block
        a, b = max(offset, r0), min(offset + m, r0 + block)
        new = x[a - offset:b - offset]
        fin = np.abs(new[np.isfinite(new)])
        s = scale_of(float(fin.max()) if fin.size else 0.0, fmt)
        old = scales[blk] if r0 < offset else 0.0
        s = max(s, old)
        if r0 < offset and s > old:
            ratio = float(np.float32(old) / np.float32(s))
            codes[r0:offset] = encode_values(decode_codes(codes[r0:offset], fmt) * ratio, fmt)
        r = float(np.float32(1.0) / np.float32(s)) if s > 0 else 0.0
        with np.errstate(invalid="ignore"):
            y = new * r
        y = np.where(np.isnan(y), 0.0, y)
        codes[a:b] = encode_values(y, fmt)
        scales[blk] = s


def values(codes, scales, block, fmt):
    """Row values [rows][D] (float64) of codes [rows][D]."""
    return decode_codes(codes, fmt) * np.repeat(scales, block)[:len(codes), None]


def attention(q, K, V, tau):
    """Softmax attention of one head in 64 bits: out [D], lse (empty: zeros, -inf)."""
    if len(K) == 0:
        return np.zeros(q.shape[-1]), -np.inf
    s = K @ q * tau
    m = s.max()
    p = np.exp(s - m)
    return (p @ V) / p.sum(), m + np.log(p.sum())


EPS = 2.0 ** -24   # half a step of fp32, relative


def attention_tolerance(q, K, V, tau):
    """Bounds on |out - exact| and |lse - exact| of fp32 arithmetic: a logit is a D-term sum of products held to 24
    bits, off by at most d = (D + 8) EPS sum|q k| tau; weights then move by a factor within exp(+-2d), the values' mean
    by at most that times their spread, and the sums over the rows add one rounding per row."""
    n, D = K.shape if len(K) else (0, len(q))
    if n == 0:
        return 0.0, 0.0
    d = (D + 8) * EPS * float((np.abs(K) @ np.abs(q)).max()) * tau
    rows = (n + 64) * EPS
    lse = float(np.abs(K @ q * tau).max()) + np.log(n)
    return float(np.abs(V).max()) * (4 * d + 2 * rows) + 1e-37, d + rows + 2 * EPS * lse
