"""Oracle for the 8-bit paged cache: written, read and attended over, in float64.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``).

A value is an e4m3 code (sign, 4 exponent bits with bias 7, 3 mantissa bits;
0x7F and 0xFF are NaN, no infinity, largest 448) times the scale of its page
and KV head, 2^e or 0: e the least integer >= -126 with amax <= 448 * 2^e.
Every step of writing is exact in float64 but the rounding to a code, which is
to nearest, ties to the even code; at scale 2^120 codes end at 240, so that what
they stand for is an fp32 number.
"""
from __future__ import annotations

from typing import Optional, Sequence, Tuple

import numpy as np

MAX = 448.0


def _table() -> np.ndarray:
    v = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        x = np.nan if (b & 127) == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[b] = -x if b & 128 else x
    return v


VALUE = _table()
_POS = VALUE[:127]                      # 0 .. 448, increasing


def encode(x: np.ndarray) -> np.ndarray:
    """Codes of x, |x| <= 448 (rounded to nearest even code); not finite -> 0x7F."""
    x = np.asarray(x, np.float64)
    ok = np.isfinite(x)
    a = np.where(ok, np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(_POS, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dh, dl = _POS[hi] - a, a - _POS[lo]
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = np.where(_POS[hi] == a, hi, code).astype(np.uint8)
    code = np.where(np.signbit(x) & ok, code | 128, code)
    return np.where(ok, code, 0x7F).astype(np.uint8)


def scale_of(amax: float) -> float:
    if amax == 0.0:
        return 0.0
    e = -126
    while amax > MAX * 2.0 ** e:
        e += 1
    return 2.0 ** e


def append(codes: np.ndarray, scale: np.ndarray, table: np.ndarray, lens: Sequence[int], rows: Sequence[int],
           x: np.ndarray) -> None:
    """x [rows][Hkv][d] into codes [pages][Hkv][page][d] and scale [pages][Hkv], in place."""
    page, Hkv = codes.shape[2], codes.shape[1]
    x = np.asarray(x, np.float64)
    at = 0
    for r, (n, m) in enumerate(zip(lens, rows)):
        lo = max(n - m, 0)
        for j in range(lo // page, -(-n // page) if n > lo else 0):
            p, a, b = table[r][j], max(lo - j * page, 0), min(n - j * page, page)
            src = x[at + (j * page + a) - (n - m):at + (j * page + b) - (n - m)]
            for g in range(Hkv):
                y = src[:, g]
                fin = np.abs(y[np.isfinite(y)])
                old = float(scale[p, g]) if a > 0 else 0.0
                now = max(old, scale_of(float(fin.max()) if fin.size else 0.0))
                s = now if now > 0 else 1.0
                if now > old:
                    codes[p, g, :a] = encode(VALUE[codes[p, g, :a]] * old / s)
                with np.errstate(invalid="ignore", over="ignore"):
                    # (at the largest scale a code of 256 would stand for 2^128, which is no fp32 number)
                    top = 240.0 if s == 2.0 ** 120 else MAX
                    codes[p, g, a:b] = encode(np.where(np.isfinite(y), np.clip(y / s, -top, top), y))
                scale[p, g] = now
        at += m


def gather(codes: np.ndarray, scale: np.ndarray, ids: Sequence[int], n: int, g: int) -> np.ndarray:
    """The first n tokens of KV head g of a request with pages `ids`: [n][d]."""
    page, d = codes.shape[2], codes.shape[3]
    k = -(-n // page)
    ids = np.asarray(ids[:k], np.int64)
    return (VALUE[codes[ids, g]] * scale[ids, g].astype(np.float64)[:, None, None]).reshape(k * page, d)[:n]


def attention(q: np.ndarray, K: np.ndarray, V: np.ndarray, first: Optional[int],
              scale: float) -> Tuple[np.ndarray, np.ndarray, np.ndarray]:
    """Rows q [m][d] over tokens K, V [n][d]; row i sees tokens 0 .. first + i (all with
    first None).  Returns out [m][d], lse [m], and sum p |V| / sum p [m][d]."""
    m, n = q.shape[0], K.shape[0]
    out, absv, lse = np.zeros(q.shape), np.zeros(q.shape), np.full(m, -np.inf)
    for i in range(m):
        k = n if first is None else min(n, max(0, first + i + 1))
        if k == 0:
            continue
        x = (K[:k] @ q[i]) * scale
        top = x.max()
        p = np.exp(x - top)
        out[i], absv[i] = p @ V[:k] / p.sum(), p @ np.abs(V[:k]) / p.sum()
        lse[i] = top + np.log(p.sum())
    return out, lse, absv
