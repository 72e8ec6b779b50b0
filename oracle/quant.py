"""Oracle of the KV cache in 8 bits -- TEST INFRASTRUCTURE ONLY (numpy, 64 bits, no code of the library's).

A cache block of rows shares one scale byte s; a code c stands for c * 2^(s - 127), and for 0 where s is 0. Codes are bytes:
e4m3 (sign, 4 exponent bits with bias 7, 3 mantissa bits; 0x7F and 0xFF NaN; largest 448) or two's complement int8 (-128
stands for NaN).
"""
from __future__ import annotations

import numpy as np

LARGEST = {"e4m3": 448.0, "int8": 127.0}
NAN_CODE = {"e4m3": 0x7F, "int8": 0x80}


def _table(fmt: str) -> np.ndarray:
    """Value of every byte."""
    c = np.arange(256)
    if fmt == "int8":
        v = c.astype(np.uint8).view(np.int8).astype(np.float64)
        v[0x80] = np.nan
        return v
    e, m, sign = (c >> 3) & 15, c & 7, np.where(c >= 128, -1.0, 1.0)
    v = sign * np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[[0x7F, 0xFF]] = np.nan
    return v


TABLE = {f: _table(f) for f in LARGEST}


def encode(x: np.ndarray, fmt: str) -> np.ndarray:
    """Finite x of at most the largest magnitude -> nearest code, ties to the one with an even last bit."""
    x = np.asarray(x, np.float64)
    assert np.all(np.abs(x) <= LARGEST[fmt])
    n = 128 if fmt == "int8" else 127                       # magnitudes by code, ascending
    mags = np.arange(128.0) if fmt == "int8" else TABLE[fmt][:127]
    a = np.abs(x)
    hi = np.minimum(np.searchsorted(mags, a), n - 1)        # first magnitude >= a
    lo = np.maximum(hi - 1, 0)
    to_lo, to_hi = a - mags[lo], mags[hi] - a
    pick = np.where((to_lo < to_hi) | ((to_lo == to_hi) & (lo % 2 == 0)), lo, hi)
    pick = np.where(mags[hi] == a, hi, pick)
    neg = np.signbit(x)
    if fmt == "int8":
        return np.where(neg, -pick, pick).astype(np.int8).view(np.uint8)
    return (pick | np.where(neg, 0x80, 0)).astype(np.uint8)


def _below(x: np.ndarray, s: int, fmt: str) -> np.ndarray:
    """Codes' values that stand for 2^128 or more are not written: magnitudes cut to the largest code that stands for less."""
    t = TABLE[fmt]
    t = t[np.isfinite(t)]
    most = t[t * 2.0 ** (s - 127.0) < 2.0 ** 128].max()
    return np.clip(x, -most, most)


def need(top: float, fmt: str) -> int:
    """The smallest s >= 1 with top <= largest * 2^(s - 127); 0 for top = 0."""
    if top == 0:
        return 0
    s = 1
    while top > LARGEST[fmt] * 2.0 ** (s - 127):
        s += 1
    return s


def values(codes: np.ndarray, scales: np.ndarray, block: int, fmt: str) -> np.ndarray:
    """codes u8 [..., rows, d], scales u8 [..., ceil(rows / block)] -> fp64 values."""
    s = np.repeat(scales, block, axis=-1)[..., :codes.shape[-2]].astype(np.float64)
    return TABLE[fmt][codes] * np.where(s > 0, 2.0 ** (s - 127), 0.0)[..., None]


def write(codes: np.ndarray, scales: np.ndarray, x: np.ndarray, start: int, count: int, block: int, fmt: str) -> None:
    """Rows x[:count] of one head to positions start .. of codes [capacity][d], scales [blocks], in place."""
    cap = codes.shape[0]
    if not 0 <= start < cap:
        return
    count = min(max(count, 0), len(x), cap - start)
    end = start + count
    for b in range(start // block, -(-end // block) if count else 0):
        r0, r1 = max(start, b * block), min(end, (b + 1) * block)
        new = x[r0 - start:r1 - start].astype(np.float64)
        fine = np.isfinite(new).all(1)
        s = need(float(np.abs(new[fine]).max()) if fine.any() else 0.0, fmt)
        if b * block < start:
            old = int(scales[b])
            front = codes[b * block:start]
            s = max(s, old)
            if s > old:
                v = TABLE[fmt][front] * (2.0 ** (old - s) if old else 0.0)
                nan = np.isnan(v)
                codes[b * block:start] = np.where(nan, front, encode(_below(np.where(nan, 0.0, v), s, fmt), fmt))
        scales[b] = s
        new[~fine] = 0.0
        codes[r0:r1] = np.where(fine[:, None], encode(_below(new * 2.0 ** (127 - s) if s else new, s, fmt), fmt), NAN_CODE[fmt])


def attend(q, k, v, keys, scale=None):
    """One query row q [d] over rows `keys` of k, v [rows][d] in 64 bits. Returns (O [d], lse, A [d], Z): the weighted mean of
    |v| and the largest sum of |q_d k_d| times the scale among the keys, from which bounds of a 32-bit evaluation follow."""
    q, d = q.astype(np.float64), q.shape[0]
    scale = 1 / np.sqrt(d) if scale is None else scale
    if len(keys) == 0:
        return np.zeros(d), -np.inf, np.zeros(d), 0.0
    kk, vv = k[keys], v[keys]
    with np.errstate(invalid="ignore"):
        z = kk @ q * scale
        m = z.max()
        w = np.exp(z - m)
        L = w.sum()
        return (w @ vv) / L, m + np.log(L), (w @ np.abs(vv)) / L, float(np.nanmax(np.abs(kk) @ np.abs(q)) * scale)
