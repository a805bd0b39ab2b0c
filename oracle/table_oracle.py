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


def row_exponent(amax: np.ndarray) -> np.ndarray:
    """Least k with amax <= 2688 * 2^k, in [-110, 116]; 0 for a row of zeros."""
    amax = np.asarray(amax, np.float64)
    k = np.frexp(amax / 2688.0)[1].astype(np.int64) + 1      # (one too many at least)
    for _ in range(3):
        k = np.where(amax <= 2688.0 * 2.0 ** (k - 1.0), k - 1, k)
    return np.where(amax > 0, np.clip(k, -110, 116), 0)


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
    good = np.isfinite(b).all(2)
    b = np.where(good[:, :, None], b, 0.0)
    amax = np.abs(b).max(2)
    exps = np.zeros(R, np.int64)
    if fmt == "e4m3":
        exps = row_exponent(amax.max(1)) if row_exps is None else np.asarray(row_exps)
        unit = 2.0 ** exps.astype(np.float64)[:, None]
        scales = nearest((amax / 6 / unit).reshape(-1), _E4M3).reshape(amax.shape)
        step = _E4M3[scales] * unit
        bad = 0x7F
    else:
        e = np.where(amax > 0, np.maximum(np.frexp(amax)[1].astype(np.int64) - 3, -126), -126)
        scales, step, bad = e + 127, 2.0 ** e.astype(np.float64), 0xFF
    ratio = np.abs(b) / np.where(step > 0, step, 1.0)[:, :, None]
    q = np.where((step > 0)[:, :, None], nearest(ratio.reshape(-1), E2M1).reshape(b.shape), 0)
    codes = (q + 8 * np.signbit(b)).astype(np.uint8)
    codes[~good] = 0
    scales = np.where(good, scales, bad).astype(np.uint8)
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
