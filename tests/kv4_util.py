"""The 4-bit cache in 64-bit NumPy, element by element from its definition (used by
the tests of the calls that write and read it)."""
from __future__ import annotations

import numpy as np

from kv8_util import EPS

FORMATS = ("fp4", "int4")
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TINY, MOST = 2.0 ** -126, 2.0 ** 126
F = np.float32


def place(d: int, fmt: str) -> tuple[int, int]:
    """The byte and the shift in it of dimension d's code."""
    if fmt == "fp4":
        return d // 2, 4 * (d % 2)
    p = 8 * (d // 8) + (d % 8) // 2 + 4 * (d % 2)     # its nibble
    return p // 2, 4 * (p % 2)


def pack(codes: np.ndarray, fmt: str) -> np.ndarray:
    """Codes [..][D] as bytes [..][D / 2]."""
    D = codes.shape[-1]
    out = np.zeros(codes.shape[:-1] + (D // 2,), np.uint8)
    for d in range(D):
        b, s = place(d, fmt)
        out[..., b] |= (codes[..., d] << s).astype(np.uint8)
    return out


def unpack(data: np.ndarray, fmt: str) -> np.ndarray:
    D = 2 * data.shape[-1]
    return np.stack([(data[..., place(d, fmt)[0]] >> place(d, fmt)[1]) & 15 for d in range(D)], axis=-1)


def bf16_grid(x: float, up: bool) -> float:
    """x rounded up or down to a bf16 (of a normal magnitude; 0 stays)."""
    if x == 0:
        return 0.0
    step = 2.0 ** (max(np.frexp(abs(x))[1], -125) - 8)
    return float((np.ceil if up else np.floor)(x / step) * step)


def encode_row(x: np.ndarray, fmt: str) -> tuple[np.ndarray, int]:
    """A row x [D] (float64): its codes and its word."""
    D = len(x)
    fin = np.isfinite(x)
    x0 = np.where(np.isnan(x), 0.0, x)
    codes = np.zeros(D, np.uint8)
    if fmt == "fp4":
        word = 0
        for g in range(4):
            at = slice(g * D // 4, (g + 1) * D // 4)
            amax = float(np.abs(x[at][fin[at]]).max(initial=0.0))
            if amax == 0:
                continue
            e = -126
            while amax > 7.0 * 2.0 ** e and e < 125:
                e += 1
            word |= (e + 127) << 8 * g
            a = np.minimum(np.abs(x0[at]) / 2.0 ** e, 6.0)
            hi = np.clip(np.searchsorted(E2M1, a), 0, 7)       # first code with magnitude >= a
            lo = np.maximum(hi - 1, 0)
            dl, dh = a - E2M1[lo], E2M1[hi] - a
            c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
            codes[at] = c | np.where(np.signbit(x0[at]), 8, 0)
        return codes, word
    v = np.clip(x[fin], -MOST, MOST)
    lo, hi = (float(v.min()), float(v.max())) if v.size else (0.0, 0.0)
    m = bf16_grid(lo, False)
    d = F(F(hi) - F(m))
    s = F(bf16_grid(max(float(d / F(15)), TINY), True)) if d > 0 else F(0)
    r = F(1) / s if s > 0 else F(0)
    with np.errstate(invalid="ignore", over="ignore"):
        y = (x0.astype(F) - F(m)).astype(np.float64) * float(r)
    y = np.where(np.isnan(y), 0.0, y)
    bits = [int(np.array(t, F).view(np.uint32)) for t in (s, F(m))]
    return np.clip(np.rint(y), 0, 15).astype(np.uint8), bits[0] >> 16 | bits[1]


def row_values(codes: np.ndarray, word: np.ndarray, fmt: str) -> np.ndarray:
    """Values (float64) of codes [..][D] under words [..]; int4's are rounded to floats, as the call gives them."""
    D = codes.shape[-1]
    word = word.astype(np.uint32)
    if fmt == "fp4":
        byte = np.stack([(word >> 8 * g) & 255 for g in range(4)], axis=-1).astype(np.int64)
        s = np.where(byte > 0, 2.0 ** (byte - 127.0), 0.0).repeat(D // 4, axis=-1)
        return E2M1[codes & 7] * np.where(codes & 8, -1.0, 1.0) * s
    s, m = parts(word)
    return (codes * s[..., None] + m[..., None]).astype(F).astype(np.float64)


def parts(word: np.ndarray):
    """int4's steps and bases."""
    word = word.astype(np.uint32)
    return tuple(np.ascontiguousarray(t).view(F).astype(np.float64).reshape(word.shape)
                 for t in (word << np.uint32(16), word & np.uint32(0xFFFF0000)))


def exact_values(codes: np.ndarray, word: np.ndarray, fmt: str) -> np.ndarray:
    """The same, int4's without the rounding."""
    if fmt == "fp4":
        return row_values(codes, word, fmt)
    s, m = parts(word)
    return codes * s[..., None] + m[..., None]


def bulk(codes: np.ndarray, word: np.ndarray, fmt: str) -> np.ndarray:
    """What the sums of a product over these rows hold at most in place of each value: int4's codes meet the products
    apart from their base, and the two cancel."""
    if fmt == "fp4":
        return np.abs(row_values(codes, word, fmt))
    s, m = parts(word)
    return codes * s[..., None] + np.abs(m)[..., None]


def attention_tolerance(q, K, V, Kb, Vb, tau):
    """Bounds on |out - exact| and |lse - exact| of fp32 arithmetic over values K, V whose sums hold Kb, Vb (bulk):
    a logit is a D-term sum of products held to 24 bits, off by at most d = (D + 8) EPS sum|q| Kb tau; weights then move
    by a factor within exp(+-2d) and move the mean by at most that times the values' spread; the sums over the rows add
    one rounding of what they hold per row."""
    n, D = K.shape if len(K) else (0, len(q))
    if n == 0:
        return 0.0, 0.0
    d = (D + 8) * EPS * float((Kb @ np.abs(q)).max()) * tau
    rows = (n + 64) * EPS
    lse = float(np.abs(K @ q * tau).max()) + np.log(n)
    return float(np.abs(V).max()) * 4 * d + 2 * rows * float(Vb.max()) + 1e-37, d + rows + 2 * EPS * lse


def random_cache(rng, shape, D, fmt):
    """Codes [shape][D], words [shape] of one tensor: every code, scales spread over three orders of magnitude."""
    codes = rng.integers(0, 16, shape + (D,)).astype(np.uint8)
    if fmt == "fp4":
        byte = rng.integers(124, 129, shape + (4,)).astype(np.uint32)
        return codes, byte[..., 0] | byte[..., 1] << 8 | byte[..., 2] << 16 | byte[..., 3] << 24
    s = (np.exp(rng.uniform(-3, 0, shape)) * 0.3).astype(F)
    m = (s * rng.uniform(-12, -3, shape)).astype(F)
    sb, mb = (np.ascontiguousarray(t).view(np.uint32) & np.uint32(0xFFFF0000) for t in (s, m))
    return codes, sb >> np.uint32(16) | mb


def records(ck, cv, fmt):
    """K's and V's codes as records [..][D] of bytes."""
    return np.concatenate([pack(ck, fmt), pack(cv, fmt)], axis=-1)
