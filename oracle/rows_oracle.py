"""The operators around the head's product in 64 bits, written from their formulas.

  norm, norm_grads   layer norm of rows, and its gradients
  encode8, decode8   rows in e4m3 with a scale for each block of 128 columns, and the
                     values they stand for
  product8           logits over kept rows of such a table
  shape              logits with penalties, biases and masks

Test infrastructure only: plain and slow, numpy alone.
"""
from __future__ import annotations

import numpy as np

from .table_oracle import e4m3_table, nearest

_E4M3 = e4m3_table()


def norm(x, weight=None, bias=None, eps=1e-5, centre=True):
    """(y, mean, rstd) of rows x [R, d]."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1) if centre else np.zeros(x.shape[0])
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if weight is not None:
        y = y * np.asarray(weight, np.float64)
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    return y, mean, rstd


def norm_grads(d_out, x, weight, mean, rstd):
    """(d_x, d_weight, d_bias); mean None: not centred."""
    dy, x = np.asarray(d_out, np.float64), np.asarray(x, np.float64)
    r = np.asarray(rstd, np.float64)[:, None]
    n = (x if mean is None else x - np.asarray(mean, np.float64)[:, None]) * r
    g = dy if weight is None else dy * np.asarray(weight, np.float64)
    d = max(x.shape[1], 1)
    inner = g - n * ((g * n).sum(1, keepdims=True) / d)
    if mean is not None:
        inner = inner - g.sum(1, keepdims=True) / d
    return r * inner, (dy * n).sum(0), dy.sum(0)


def encode8(x, block_rows=1):
    """x [R, d] -> (codes uint8 [R, d], scales float32 [row blocks, column blocks])."""
    x = np.asarray(x, np.float64)
    R, d = x.shape
    rb, cb = -(-R // block_rows), -(-d // 128)
    codes, scales = np.zeros((R, d), np.uint8), np.zeros((rb, cb), np.float32)
    for i in range(rb):
        for b in range(cb):
            at = (slice(i * block_rows, (i + 1) * block_rows), slice(128 * b, 128 * b + 128))
            v = x[at]
            if not np.isfinite(v).all():
                scales[i, b] = np.nan
                continue
            amax = np.float32(np.abs(v).max())
            s = max(np.float32(amax / np.float32(448)), np.float32(2.0 ** -126))
            scales[i, b] = s
            q = nearest((np.abs(v) / np.float64(s)).reshape(-1), _E4M3).reshape(v.shape)
            codes[at] = (q + 128 * np.signbit(v)).astype(np.uint8)
    return codes, scales


def decode8(codes, scales, block_rows=1):
    """The values that codes [R, d] and scales stand for."""
    c = np.asarray(codes)
    v = np.append(_E4M3, np.nan)[c & 127] * np.where(c >= 128, -1.0, 1.0)
    f = np.repeat(np.asarray(scales, np.float64), block_rows, axis=0)[:c.shape[0]]
    return v * np.repeat(f, 128, axis=1)[:, :c.shape[1]]


def held8(x, block_rows=1):
    return decode8(*encode8(x, block_rows), block_rows)


def product8(h, table, ids=None, bias=None):
    """Logits of h [R, d], held in e4m3 blocks of one row, over rows `ids` of the decoded
    table [V, d]; and the sums of the products' magnitudes."""
    x, w = held8(h), np.asarray(table, np.float64)
    w = w if ids is None else w[ids]
    y = x @ w.T
    if bias is not None:
        b = np.asarray(bias, np.float64)
        y = y + (b if ids is None else b[ids])
    return y, np.abs(x) @ np.abs(w).T


def shape(z, V, ids=None, history=None, lengths=None, prompts=None, repetition=None,
          frequency=None, presence=None, bias_ids=None, bias_values=None, mask=None,
          mask_rows=None, dtype=np.float64):
    """z [R, n] with penalties, biases and masks, each step rounded to `dtype`."""
    z = np.asarray(z, dtype).copy()
    R, n = z.shape
    ids = np.arange(V) if ids is None else np.asarray(ids)
    column = {int(v): j for j, v in enumerate(ids)}
    for r in range(R):
        if history is not None:
            length = len(history[r]) if lengths is None else min(max(int(lengths[r]), 0), len(history[r]))
            prompt = 0 if prompts is None else int(prompts[r])
            seen, said = set(), {}
            for i in range(length):
                v = int(history[r][i])
                if v in column:
                    seen.add(v)
                    if i >= prompt:
                        said[v] = said.get(v, 0) + 1
            for v in seen:
                j = column[v]
                if repetition is not None:
                    rho = dtype(repetition[r])
                    z[r, j] = z[r, j] / rho if z[r, j] > 0 else z[r, j] * rho
                if v in said:
                    if frequency is not None:
                        z[r, j] = z[r, j] - dtype(frequency[r]) * dtype(said[v])
                    if presence is not None:
                        z[r, j] = z[r, j] - dtype(presence[r])
        if bias_ids is not None:
            sums = {}
            for v, b in zip(bias_ids[r], bias_values[r]):
                if int(v) in column:
                    sums[int(v)] = dtype(sums.get(int(v), dtype(0)) + dtype(b))
            for v, b in sums.items():
                z[r, column[v]] = z[r, column[v]] + b
        if mask is not None:
            m = r if mask_rows is None else int(mask_rows[r])
            if m >= 0:
                words = np.asarray(mask[m]).astype(np.int64) & 0xFFFFFFFF
                z[r, (words[ids >> 5] >> (ids & 31)) & 1 == 0] = -np.inf
    return z
