"""Norms of queries and keys with the rotation, their gradients, the 8-bit cache and attention over it, in float64 numpy.
Written from the formulas, row by row."""
from __future__ import annotations

import math
from typing import Optional, Tuple

import numpy as np

TOP, LOWEST = 448.0, -64


def rope_frequencies(theta: float, rotary: int, scaling: str = "none", factor: float = 1.0, original_len: int = 1,
                     beta_fast: float = 32.0, beta_slow: float = 1.0) -> Tuple[np.ndarray, float]:
    """Frequencies [rotary / 2] and the factor on the rotated pairs."""
    w = np.array([theta ** (-2.0 * d / rotary) for d in range(rotary // 2)])
    if scaling == "linear":
        return w / factor, 1.0
    if scaling == "yarn":
        out = []
        for f in w:
            turns = original_len * f / (2 * math.pi)
            gamma = min(max((turns - beta_slow) / (beta_fast - beta_slow), 0.0), 1.0)
            out.append((1 - gamma) * f / factor + gamma * f)
        return np.array(out), 0.1 * math.log(factor) + 1.0
    return w, 1.0


def _members(rotary: int, style: int):
    half = rotary // 2
    d = np.arange(half)
    return (d, d + half) if style == 0 else (2 * d, 2 * d + 1)


def rotate(x: np.ndarray, pos: np.ndarray, freq: np.ndarray, factor: float, style: int) -> np.ndarray:
    """x [..., H, D] at positions pos [...]; the first 2 * len(freq) elements turn."""
    a, c = _members(2 * len(freq), style)
    t = np.asarray(pos, dtype=np.float64)[..., None, None] * freq
    y = np.array(x, dtype=np.float64)
    y[..., a] = factor * (x[..., a] * np.cos(t) - x[..., c] * np.sin(t))
    y[..., c] = factor * (x[..., c] * np.cos(t) + x[..., a] * np.sin(t))
    return y


def norm_rope(x: np.ndarray, gain: Optional[np.ndarray], eps: float, pos, freq, factor, style) -> np.ndarray:
    y = np.asarray(x, dtype=np.float64)
    if gain is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * gain
    return rotate(y, pos, freq, factor, style)


def norm_rope_backward(x, gain, eps, pos, freq, factor, style, dy):
    """(dx, dgain or None)."""
    dn = rotate(np.asarray(dy, dtype=np.float64), pos, -np.asarray(freq), factor, style)      # the transpose of a turn is the turn back
    if gain is None:
        return dn, None
    x = np.asarray(x, dtype=np.float64)
    root = np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u = x / root
    dgain = (dn * u).reshape(-1, x.shape[-1]).sum(0)
    return (dn * gain - u * (dn * gain * u).mean(-1, keepdims=True)) / root, dgain


# ---------------------------------------------------------------------------------------------- e4m3
def code_value(code: int) -> float:
    """s eeee mmm: bias 7, no infinities, s1111111 is NaN."""
    e, m = (code >> 3) & 15, code & 7
    if e == 15 and m == 7:
        return math.nan
    x = math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)
    return -x if code & 128 else x


VALUES = np.array([code_value(c) for c in range(256)])


def to_code(x: np.ndarray) -> np.ndarray:
    """Nearest code, ties to the even one; beyond the range the largest; NaN to NaN."""
    x = np.asarray(x, dtype=np.float64)
    grid = VALUES[:127]                                            # 0 .. 448, ascending with the code
    a = np.minimum(np.abs(x), TOP)
    hi = np.clip(np.searchsorted(grid, np.nan_to_num(a)), 1, 126)
    lo = hi - 1
    d_lo, d_hi = a - grid[lo], grid[hi] - a
    c = np.where((d_hi < d_lo) | ((d_hi == d_lo) & (hi % 2 == 0)), hi, lo)
    c = np.where(np.signbit(x), c | 128, c)
    return np.where(np.isnan(x), 127, c).astype(np.uint8)


def page_exponent(x: np.ndarray) -> int:
    """e of the smallest 2^e >= 2^-64 with max|x| <= 448 * 2^e, over the finite values."""
    a = np.abs(x[np.isfinite(x)])
    top = float(a.max()) if a.size else 0.0
    e = LOWEST
    while top > math.ldexp(TOP, e):
        e += 1
    return e


def append(rows, codes, scale, table, prefix, count, page):
    """rows [B,W,Hkv,D] -> new (codes, scale, slots); codes u8 [pages,Hkv,page,D], scale [pages,Hkv]."""
    codes, scale = codes.copy(), scale.astype(np.float64).copy()
    B, W, H, D = rows.shape
    slots = np.full((B, W), -1, dtype=np.int64)
    for b in range(B):
        n = W if count is None else min(max(int(count[b]), 0), W)
        P = int(prefix[b])
        for j in range(P // page, -(-(P + n) // page) if n else 0):
            if j >= table.shape[1] or not 0 <= table[b, j] < codes.shape[0]:
                continue
            at = int(table[b, j])
            for i in range(max(P, j * page), min(P + n, (j + 1) * page)):
                slots[b, i - P] = at * page + i - j * page
            for h in range(H):
                held = [VALUES[codes[at, h, r]] * scale[at, h] for r in range(max(0, min(P - j * page, page)))]
                held += [np.asarray(rows[b, i - P, h], dtype=np.float64) for i in range(max(P, j * page), min(P + n, (j + 1) * page))]
                held = np.array(held)
                e = page_exponent(held)
                codes[at, h, : len(held)] = to_code(held * 2.0 ** -e)
                scale[at, h] = 2.0 ** e
    return codes, scale, slots


def attention(q, k_codes, k_scale, v_codes, v_scale, table, prefix, softmax_scale):
    """(out [B,W,Hq,D], average of |v| under the same weights): the second is what errors of single weights are relative to."""
    B, W, Hq, D = q.shape
    Hkv, page = k_codes.shape[1], k_codes.shape[2]
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(B):
        n = int(prefix[b]) + W
        pages = table[b, : -(-n // page)].astype(np.int64)
        k = (VALUES[k_codes[pages]] * np.asarray(k_scale, dtype=np.float64)[pages][:, :, None, None]).transpose(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :n]
        v = (VALUES[v_codes[pages]] * np.asarray(v_scale, dtype=np.float64)[pages][:, :, None, None]).transpose(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :n]
        for h in range(Hq):
            g = h * Hkv // Hq
            for i in range(W):
                m = int(prefix[b]) + i + 1
                s = k[g, :m] @ np.asarray(q[b, i, h], dtype=np.float64) * softmax_scale
                p = np.exp(s - s.max())
                p /= p.sum()
                out[b, i, h], size[b, i, h] = p @ v[g, :m], p @ np.abs(v[g, :m])
    return out, size
