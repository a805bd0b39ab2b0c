"""The operators on a vocabulary table in 64 bits, written from their formulas.

  encode / decode   rows in e2m1 codes with block scales, and the values they
                    stand for
  terms             a row as a sum of 4-bit terms
  product           logits over kept rows of a table held in 4 bits
  lookup, gradient  rows by token, and the table's gradient

Test infrastructure only: plain and slow, numpy alone.
"""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = {"e8m0": 32, "e4m3": 16}


def e4m3_table() -> np.ndarray:
    """The 127 values >= 0 of e4m3 (code order): 4 exponent bits of bias 7, 3 of mantissa."""
    v = []
    for code in range(127):
        e, m = code >> 3, code & 7
        v.append(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(v)


_E4M3 = e4m3_table()


def nearest(values: np.ndarray, grid: np.ndarray) -> np.ndarray:
    """Index of the grid entry nearest to each value; of two as near, the even index;
    values past the last entry take it."""
    hi = np.clip(np.searchsorted(grid, values), 1, len(grid) - 1)
    lo = hi - 1
    d_lo, d_hi = values - grid[lo], grid[hi] - values
    return np.where((d_hi < d_lo) | ((d_hi == d_lo) & (hi % 2 == 0)), hi, lo)


def row_exponent(amax: float) -> int:
    """Least k with amax <= 2688 * 2^k, in [-110, 116]; 0 for a row of zeros."""
    if amax == 0:
        return 0
    k = -400
    m, e = np.frexp(amax / 2688.0)         # amax / 2688 = m 2^e, m in [0.5, 1)
    for k in (int(e) - 2, int(e) - 1, int(e), int(e) + 1):
        if amax <= 2688.0 * 2.0 ** k:
            break
    return int(min(116, max(-110, k)))


def encode(x, fmt: str, row_exps=None):
    """x [R, d] (any float type) -> (codes uint8 [R, dp] of 4 bits each, scale bytes uint8
    [R, blocks], row exponents int [R]).  dp: d up to a whole 32 columns."""
    x = np.asarray(x, dtype=np.float64)
    R, d = x.shape
    bs, dp = BLOCK[fmt], -(-d // 32) * 32
    nb = -(-d // bs)
    b = np.zeros((R, dp))
    b[:, :d] = x
    b = b.reshape(R, dp // bs, bs)
    codes = np.zeros((R, dp // bs, bs), np.uint8)
    scales = np.zeros((R, dp // bs), np.uint8)
    exps = np.zeros(R, np.int64)
    for r in range(R):
        good = np.isfinite(b[r]).all(1)
        amax = np.where(good, np.abs(np.where(np.isfinite(b[r]), b[r], 0)).max(1), 0)
        if fmt == "e4m3":
            exps[r] = row_exponent(amax.max()) if row_exps is None else row_exps[r]
        for i in range(nb):
            if not good[i]:
                scales[r, i] = 0x7F if fmt == "e4m3" else 0xFF
                continue
            if fmt == "e4m3":
                scales[r, i] = nearest(np.array([amax[i] / 6 / 2.0 ** exps[r]]), _E4M3)[0]
                step = _E4M3[scales[r, i]] * 2.0 ** exps[r]
            else:
                e = max(int(np.frexp(amax[i])[1]) - 3, -126) if amax[i] > 0 else -126
                scales[r, i] = e + 127
                step = 2.0 ** e
            if step > 0:
                q = nearest(np.abs(b[r, i]) / step, E2M1)
                codes[r, i] = q + 8 * np.signbit(b[r, i])
            else:
                codes[r, i] = 8 * np.signbit(b[r, i])
    return codes.reshape(R, dp), scales[:, :nb], exps


def decode(codes, scales, exps, d: int, fmt: str) -> np.ndarray:
    """The values that codes [R, >= d], scale bytes and row exponents stand for, [R, d]."""
    v = np.where(codes >= 8, -1.0, 1.0) * E2M1[codes & 7]
    s = scales.astype(np.int64)
    if fmt == "e4m3":
        f = np.append(_E4M3, np.nan)[s & 127] * 2.0 ** np.asarray(exps, float)[:, None]
    else:
        f = np.where(s == 255, np.nan, 2.0 ** (np.minimum(s, 254) - 127.0))
    return v[:, :d] * np.repeat(f, BLOCK[fmt], axis=1)[:, :d]


def terms(x, fmt: str, planes: int) -> np.ndarray:
    """Sum of `planes` terms: each codes what the ones before it left of x."""
    left = np.asarray(x, dtype=np.float64)
    held, exps = np.zeros_like(left), None
    for _ in range(planes):
        c, s, e = encode(left, fmt, exps)
        exps = e if exps is None else exps
        q = decode(c, s, exps, left.shape[1], fmt)
        held, left = held + q, left - q
    return held


def unpack(packed: np.ndarray) -> np.ndarray:
    """Bytes [R, n] -> 4-bit codes [R, 2 n], the low half first."""
    out = np.empty((packed.shape[0], 2 * packed.shape[1]), np.uint8)
    out[:, 0::2], out[:, 1::2] = packed & 15, packed >> 4
    return out


def product(h, table: np.ndarray, fmt: str, planes: int, ids=None, bias=None) -> np.ndarray:
    """Logits of h [R, d] over rows `ids` of the decoded table [V, d]."""
    w = table if ids is None else table[ids]
    y = terms(h, fmt, planes) @ w.T
    if bias is not None:
        b = np.asarray(bias, np.float64)
        y = y + (b if ids is None else b[ids])
    return y


def lookup(tokens, table: np.ndarray, scale: float, padding_id: int = -1) -> np.ndarray:
    out = np.zeros((len(tokens), table.shape[1]))
    for t, v in enumerate(tokens):
        if v != padding_id and 0 <= v < table.shape[0]:
            out[t] = scale * np.asarray(table[v], np.float64)
    return out


def gradient(tokens, d_out, V: int, scale: float, padding_id: int = -1, onto=None) -> np.ndarray:
    d_out = np.asarray(d_out, np.float64)
    g = np.zeros((V, d_out.shape[1])) if onto is None else np.array(onto, np.float64)
    for t, v in enumerate(tokens):
        if v != padding_id and 0 <= v < V:
            g[v] += scale * d_out[t]
    return g
