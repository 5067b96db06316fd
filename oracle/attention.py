"""The quantised paged cache and the attention over it, in plain numpy.

Rows are written in fp32 steps where the definition is in fp32 (scales and codes
are then the same bits as any IEEE implementation's for the same fp32 row), norms,
rotations and attention in fp64.
"""
from __future__ import annotations

import numpy as np

INT8, FP8 = 0, 1
CODE_MAX = {INT8: np.float32(127.0), FP8: np.float32(448.0)}
TINY = np.float32(2.0 ** -100)


def code_values(fmt: int) -> np.ndarray:
    """The value of each of the 256 codes (fp64; e4m3 has two NaN codes)."""
    b = np.arange(256)
    if fmt == INT8:
        return np.where(b < 128, b, b - 256).astype(np.float64)
    ex, fr = (b >> 3) & 15, b & 7
    v = np.where(ex > 0, (8 + fr) * 2.0 ** (ex - 10), fr * 2.0 ** -9)
    return np.where((b & 127) == 127, np.nan, np.where(b < 128, v, -v))


def nearest_codes(y: np.ndarray, fmt: int) -> np.ndarray:
    """Codes of the values nearest to fp32 y (within the codes' range), ties to even."""
    y = y.astype(np.float64)
    if fmt == INT8:
        return np.rint(y).astype(np.int64).astype(np.uint8)
    val = code_values(FP8)[:127]                     # 0 .. 448, ascending
    a = np.abs(y)
    hi = np.clip(np.searchsorted(val, a), 1, 126)
    lo = hi - 1
    up = (a - val[lo] > val[hi] - a) | ((a - val[lo] == val[hi] - a) & (hi % 2 == 0))
    return np.where(np.signbit(y), 128, 0).astype(np.uint8) + np.where(up, hi, lo).astype(np.uint8)


def quantise(x: np.ndarray, fmt: int):
    """(codes, scales) of fp32 rows x [..., D]."""
    x = x.astype(np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        big = np.abs(x).max(-1)
        bad, none = ~np.isfinite(x).all(-1), big < TINY
        scale = np.where(none, np.float32(0), big / CODE_MAX[fmt]).astype(np.float32)
        scale = np.where(bad, np.float32(np.nan), scale)
        live = ~(bad | none)
        y = np.where(live[..., None], x, 0) / np.where(live, scale, np.float32(1))[..., None]
    codes = nearest_codes(np.clip(y, -CODE_MAX[fmt], CODE_MAX[fmt]), fmt)
    return np.where(live[..., None], codes, 0).astype(np.uint8), scale


def head_rows(x: np.ndarray, weight, eps: float, cos_sin, pos, interleaved: bool) -> np.ndarray:
    """Norm (weight None: none) and rotation (cos_sin None: none) of x [T, h, D], fp64."""
    x = x.astype(np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + np.float64(np.float32(eps))) * weight.astype(np.float64)
    if cos_sin is not None and cos_sin.shape[1]:
        R = cos_sin.shape[1]
        a = cos_sin.astype(np.float64)[pos][:, None, :]
        z = a[..., :R // 2] + 1j * a[..., R // 2:]
        x = x.copy()
        if interleaved:
            w = (x[..., 0:R:2] + 1j * x[..., 1:R:2]) * z
            x[..., 0:R:2], x[..., 1:R:2] = w.real, w.imag
        else:
            w = (x[..., :R // 2] + 1j * x[..., R // 2:R]) * z
            x[..., :R // 2], x[..., R // 2:R] = w.real, w.imag
    return x


def cache_rows(codes: np.ndarray, scale: np.ndarray, slots: np.ndarray, fmt: int) -> np.ndarray:
    """Values [n, n_kv, D] (fp64) of the slots; codes [pages, n_kv, page, D]."""
    page = codes.shape[2]
    return code_values(fmt)[codes[slots // page, :, slots % page]] * scale[slots // page, :, slots % page].astype(np.float64)[..., None]


def chain(n: int):
    """The tree words of a chain: token i sees tokens 0 .. i."""
    return [(2 << i) - 1 for i in range(n)]


def draft_attention(q, k, v, ctx: int, words, scale: float):
    """One sequence: q [n, n_q, D], k, v [len, n_kv, D] (cached, then drafted
    tokens), words [n].  Returns out, lse, and sum_p weight |v_p| (the size of the
    terms that make up out), fp64."""
    n, n_q, D = q.shape
    G = n_q // k.shape[1]
    out, lse, mag = np.zeros((n, n_q, D)), np.full((n, n_q), -np.inf), np.zeros((n, n_q, D))
    for i in range(n):
        seen = [p for p in range(k.shape[0]) if p < ctx or (int(words[i]) >> (p - ctx)) & 1 and p - ctx < n]
        if not seen:
            continue
        for h in range(n_q):
            s = (k[seen, h // G] @ q[i, h].astype(np.float64)) * scale
            top = s.max()
            e = np.exp(s - top)
            lse[i, h] = top + np.log(e.sum())
            out[i, h] = e @ v[seen, h // G] / e.sum()
            mag[i, h] = e @ np.abs(v[seen, h // G]) / e.sum()
    return out, lse, mag
