"""Oracle of the operators around a decode step's attention and logits: 64 bits, from the definitions.

Arrays come decoded (float64 / int); pages as the library keeps them (see oracle/draft.py).
"""
from __future__ import annotations

from typing import Optional

import numpy as np

E4M3_MAX = 448.0
LEAST = -96          # of the powers of two of an 8-bit cache
MOST, MOST_CODE = 120, 240.0        # the largest one, of bf16's largest numbers, and its largest code: 256 2^120 is no bf16 number


def e4m3_values() -> np.ndarray:
    """The value of each of the 256 codes, from the format's definition."""
    code = np.arange(256)
    e, m = (code >> 3) & 15, code & 7
    v = np.where(e == 0, m * 2.0 ** -9, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    v = np.where((e == 15) & (m == 7), np.nan, v)
    return np.where(code & 128, -v, v)


def e4m3(x: np.ndarray) -> np.ndarray:
    """x rounded to e4m3 (to the nearest, ties to even); up to 448 in magnitude, or not finite (NaN)."""
    with np.errstate(invalid="ignore", divide="ignore"):
        a = np.abs(np.asarray(x, dtype=np.float64))
        e = np.floor(np.log2(np.where(a > 0, a, 1.0)))
        e = np.where(2.0 ** e > a, e - 1, np.where(2.0 ** (e + 1) <= a, e + 1, e))
        step = 2.0 ** (np.maximum(e, -6) - 3)
        return np.where(np.isfinite(x), np.sign(x) * np.rint(a / step) * step, np.nan)


def quantise(x: np.ndarray):
    """[..., dim] -> (values of the codes [..., dim], exponents [...])."""
    x = np.asarray(x, dtype=np.float64)
    top = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    by = np.full(top.shape, LEAST, dtype=np.int64)
    while (top > E4M3_MAX * 2.0 ** by).any():
        by = np.where(top > E4M3_MAX * 2.0 ** by, by + 1, by)
    y = x / (2.0 ** by)[..., None]
    return e4m3(np.where((by[..., None] == MOST) & np.isfinite(x), np.clip(y, -MOST_CODE, MOST_CODE), y)), by


def commit(K, V, K_by, V_by, k, v, slots) -> None:
    """Codes' values and exponents of rows k, v [layers][T][heads][dim] into the cache's decoded arrays, in place."""
    page, e = K.shape[3], V.shape[5]
    for t, s in enumerate(slots):
        if 0 <= s < K.shape[1] * page:
            p, at = divmod(int(s), page)
            K[:, p, :, at], K_by[:, p, :, at] = quantise(k[:, t])
            V[:, p, :, at // e, :, at % e], V_by[:, p, :, at] = quantise(v[:, t])


def read(K, V, K_by: Optional[np.ndarray], V_by: Optional[np.ndarray], slots):
    """Rows (k, v) [layers][T][heads][dim] of slots; zeros where there is none."""
    layers, pages, heads, page, dim = K.shape
    e = V.shape[5]
    k, v = np.zeros((layers, len(slots), heads, dim)), np.zeros((layers, len(slots), heads, dim))
    for t, s in enumerate(slots):
        if 0 <= s < pages * page:
            p, at = divmod(int(s), page)
            k[:, t], v[:, t] = K[:, p, :, at], V[:, p, :, at // e, :, at % e]
            if K_by is not None:
                k[:, t] *= 2.0 ** K_by[:, p, :, at][..., None]
                v[:, t] *= 2.0 ** V_by[:, p, :, at][..., None]
    return k, v


def rope(x, places, inv_freq, weight=None, eps: Optional[float] = None, interleaved: bool = False) -> np.ndarray:
    """Rows [T][heads][dim], normalised (eps) and turned."""
    y = np.array(x, dtype=np.float64)
    half = len(inv_freq)
    if eps is not None:
        y /= np.sqrt((y * y).mean(-1, keepdims=True) + eps)
    if weight is not None:
        y *= weight
    for t, place in enumerate(places):
        for i, f in enumerate(inv_freq):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, half + i)
            z = (y[t, :, a] + 1j * y[t, :, b]) * np.exp(1j * (float(place) * float(f)))
            y[t, :, a], y[t, :, b] = z.real, z.imag
    return y


UNIT = 2 ** 44


def draw(row, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(answer, logp, kept tokens in order) of one row of logits, with whole weights of any size."""
    row = np.asarray(row, dtype=np.float64)
    V = row.size
    nan = np.flatnonzero(np.isnan(row))
    if nan.size:
        return int(nan[0]), 0.0, [int(nan[0])]
    order = np.argsort(-row, kind="stable")
    top = row[order[0]]
    if top == -np.inf:
        return -1, -np.inf, []
    if top == np.inf or not temperature > 0:
        return int(order[0]), 0.0, [int(order[0])]
    with np.errstate(invalid="ignore"):
        z = np.where(np.isneginf(row[order]), -np.inf, (row[order] - top) / float(temperature))
    w = [int(v) for v in np.rint(np.exp(z) * UNIT)]
    n = min(top_k, V) if top_k > 0 else V
    total = sum(w[:n])
    if top_p < 1:
        need, sums, m = int(np.ceil(max(float(top_p), 0.0) * float(total))), 0, 0
        while m < n and (m == 0 or sums < need):
            sums += w[m]
            m += 1
        n = m
    if min_p > 0:
        least = int(np.ceil(float(min_p) * UNIT))
        n = max(1, sum(v >= least for v in w[:n]))
    total = sum(w[:n])
    goal = min(int(np.floor(min(max(float(u), 0.0), 1.0) * float(total))) if u > 0 else 0, total - 1)
    sums = 0
    for i in range(n):
        sums += w[i]
        if sums > goal:
            return int(order[i]), float(z[i] - np.log(total / UNIT)), [int(v) for v in order[:n]]
    raise AssertionError("the goal is below the sum")
