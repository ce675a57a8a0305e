"""float64 CPU oracle of the quantised cache and of the attention of new tokens over a cache.

Test infrastructure only: written from the formulas of include/kvcrush.h, one row, head or page at a time, and
independent of the CUDA path.
"""
from __future__ import annotations

import numpy as np

INT8, E4M3, INT4 = 3, 4, 5
TOP = {INT8: 127.0, E4M3: 448.0, INT4: 15.0}


def e4m3_value(code: np.ndarray) -> np.ndarray:
    """Values of 8-bit floats: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7F and 0xFF are NaN."""
    c = np.asarray(code, dtype=np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * np.exp2(np.maximum(e, 1) - 7.0))
    return np.where((c & 127) == 127, np.nan, np.where(c & 128, -v, v))


_E4M3 = np.asarray([e4m3_value(i) for i in range(127)])


def round_e4m3(y: np.ndarray) -> np.ndarray:
    """The nearest 8-bit float, ties to the even code."""
    a = np.minimum(np.abs(y), 448.0)
    hi = np.searchsorted(_E4M3, a)                      # first code with value >= a
    lo = np.maximum(hi - 1, 0)
    up, down = _E4M3[hi] - a, a - _E4M3[lo]
    pick = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    return np.copysign(_E4M3[pick], y)


def quotients(x: np.ndarray, fmt: int):
    """(x / scale or (x - zero) / scale, scale, zero) of rows x [..., D] in float64."""
    x = np.asarray(x, dtype=np.float64)
    zero = x.min(-1, keepdims=True) if fmt == INT4 else np.zeros_like(x[..., :1])
    span = (x - zero).max(-1, keepdims=True) if fmt == INT4 else np.abs(x).max(-1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        y = np.where(span / TOP[fmt] >= 2.0 ** -126, (x - zero) * TOP[fmt] / span, 0.0)
    return y, span / TOP[fmt], zero


def decode(codes: np.ndarray, scales: np.ndarray, fmt: int) -> np.ndarray:
    """float64 values of codes [..., bytes] (uint8) with scales [...] or, INT4, [..., 2]."""
    s = scales.astype(np.float64)
    if fmt == INT8:
        return codes.view(np.int8).astype(np.float64) * s[..., None]
    if fmt == E4M3:
        return e4m3_value(codes) * s[..., None]
    n = np.stack([codes & 15, codes >> 4], axis=-1).reshape(codes.shape[:-1] + (2 * codes.shape[-1],)).astype(np.float64)
    return n * s[..., :1] + s[..., 1:]


def attend_row(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float):
    """One query [D] over the rows it sees, k and v [L, D]: output [D], log-sum-exp, and what a bound on the error of a
    float32 computation needs: sum of p |v| [D] and the largest sum of |q_c k_c| * scale."""
    if len(k) == 0:
        return np.zeros(v.shape[-1]), -np.inf, np.zeros(v.shape[-1]), 0.0
    x = k @ q * scale
    top = x.max()
    if top == -np.inf:
        return np.zeros(v.shape[-1]), -np.inf, np.zeros(v.shape[-1]), 0.0
    p = np.exp(x - top)
    total = p.sum()
    return p @ v / total, top + np.log(total), p @ np.abs(v) / total, float((np.abs(k) @ np.abs(q)).max() * scale)


def page_bounds(k: np.ndarray, page_size: int):
    """(lo, hi) [pages, D] of the keys k [L, D] of one head."""
    pages = [k[a:a + page_size] for a in range(0, len(k), page_size)]
    return np.asarray([p.min(0) for p in pages]), np.asarray([p.max(0) for p in pages])


def page_scores(q: np.ndarray, lo: np.ndarray, hi: np.ndarray) -> np.ndarray:
    """Scores of pages for the query heads q [G, D] of one group."""
    out = np.zeros(len(lo))
    up, down = np.where(q > 0, q, 0).sum(0), np.where(q < 0, q, 0).sum(0)
    for p in range(len(lo)):
        out[p] = sum(hi[p, c] * up[c] for c in range(q.shape[1]) if up[c]) + sum(lo[p, c] * down[c] for c in range(q.shape[1]) if down[c])
    return out


def choose_pages(scores: np.ndarray, budget: int, keep_initial: int, keep_recent: int) -> np.ndarray:
    """Pages in order of choice: by decree, then by score; ties to the lower page.  Ascending."""
    n = len(scores)
    s = np.where(np.isnan(scores), np.inf, scores)
    decreed = [p < keep_initial or p >= n - keep_recent for p in range(n)]
    order = sorted(range(n), key=lambda p: (not decreed[p], 0.0 if decreed[p] else -s[p], p))
    return np.asarray(sorted(order[:budget]), dtype=np.int64)
