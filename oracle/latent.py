"""Attention over one latent vector a token, prompts and eviction, in plain numpy
(fp64)."""
from __future__ import annotations

import numpy as np

from .attention import head_rows


def token_rows(kv, rank: int, weight, eps: float, cos_sin, pos, interleaved: bool) -> np.ndarray:
    """Cache rows [T, rank + rot] of kv: the latent part normed, the rest turned."""
    lat = head_rows(kv[:, None, :rank], weight, eps, None, pos, interleaved)[:, 0]
    return np.concatenate([lat, head_rows(kv[:, None, rank:], None, eps, cos_sin, pos, interleaved)[:, 0]], 1)


def absorbed(q, w_k, cos_sin, pos, interleaved: bool):
    """q [T, h, D + rot] through w_k [h, D, rank], its last part turned; and the sums of
    the products' magnitudes."""
    D = w_k.shape[1]
    q = q.astype(np.float64)
    turned = head_rows(q[..., D:], None, 0.0, cos_sin, pos, interleaved)
    head = np.einsum("thd,hdr->thr", q[..., :D], w_k.astype(np.float64))
    size = np.einsum("thd,hdr->thr", np.abs(q[..., :D]), np.abs(w_k).astype(np.float64))
    return np.concatenate([head, turned], 2), np.concatenate([size, np.zeros(turned.shape)], 2)


def expanded(rows, w):
    """rows [n, rank] through w [h, D, rank], and the sums of the products' magnitudes."""
    return (np.einsum("nr,hdr->nhd", rows, w.astype(np.float64)),
            np.einsum("nr,hdr->nhd", np.abs(rows), np.abs(w).astype(np.float64)))


def softmax_rows(s, seen):
    """Weights and log-sum-exp of scores s [..., n] over the seen places (all zero, -inf where nothing is)."""
    s = np.where(seen, s, -np.inf)
    top = s.max(-1, initial=-np.inf, keepdims=True)
    top = np.where(np.isfinite(top), top, 0.0)
    e = np.where(seen, np.exp(np.where(seen, s, 0.0) - top), 0.0)
    tot = e.sum(-1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (top + np.log(tot))[..., 0]
    return e / np.where(tot > 0, tot, 1.0), lse


def tree_seen(n: int, ctx: int, words, length: int) -> np.ndarray:
    """[n, length]: places that token i sees."""
    p = np.arange(length)
    out = np.zeros((n, length), bool)
    for i in range(n):
        j = p - ctx
        out[i] = (j < 0) | ((j < n) & np.array([(int(words[i]) >> int(min(max(x, 0), 63))) & 1 for x in j], bool))
    return out


def latent_attention(q, rows, seen, w_v, scale: float):
    """One sequence: absorbed q [n, h, rank + rot], rows [len, rank + rot], seen [n, len],
    w_v [h, D, rank].  dict(out [n, h, D], lse, mass [len]; size: sum_p weight |c_p| taken through |w_v|,
    score: scale * the largest sum of the score products' magnitudes)."""
    rank = w_v.shape[2]
    q, w_v = q.astype(np.float64), w_v.astype(np.float64)
    rows = np.where(seen.any(0)[:, None], rows, 0.0)
    s = np.einsum("nhr,pr->nhp", q, rows) * scale
    w, lse = softmax_rows(s, seen[:, None, :])
    o = np.einsum("nhp,pr->nhr", w, rows[:, :rank])
    big = np.einsum("nhp,pr->nhr", w, np.abs(rows[:, :rank]))
    return dict(out=np.einsum("nhr,hdr->nhd", o, w_v), lse=lse, mass=w.sum((0, 1)),
                size=np.einsum("nhr,hdr->nhd", big, np.abs(w_v)), through=np.einsum("nhr,hdr->nhd", np.abs(o), np.abs(w_v)),
                score=abs(scale) * np.einsum("nhr,pr->nhp", np.abs(q), np.abs(rows)).max(initial=0.0))


def prompt_attention(q, k, v, r, scale: float):
    """One sequence: q [n, h, D + rot], k, v [L, g, D], r [L, rot] or None."""
    n, h, L, g = q.shape[0], q.shape[1], k.shape[0], k.shape[1]
    k = np.repeat(k.astype(np.float64), h // g, 1)
    v = np.repeat(v.astype(np.float64), h // g, 1)
    if r is not None:
        k = np.concatenate([k, np.repeat(r.astype(np.float64)[:, None], h, 1)], 2)
    seen = np.arange(L)[None, :] <= (L - n + np.arange(n))[:, None]
    used = seen.any(0)[:, None, None]
    k, v = np.where(used, k, 0.0), np.where(used, v, 0.0)
    q = q.astype(np.float64)
    w, lse = softmax_rows(np.einsum("nhd,phd->nhp", q, k) * scale, seen[:, None, :])
    return dict(out=np.einsum("nhp,phd->nhd", w, v), lse=lse, size=np.einsum("nhp,phd->nhd", w, np.abs(v)),
                score=abs(scale) * np.einsum("nhd,phd->nhp", np.abs(q), np.abs(k)).max(initial=0.0))


def evict(n: int, seq_len: int, keep: int, first: int, recent: int, mass, pos) -> np.ndarray:
    """The place that each place's token was in before, -1 from the new length on."""
    kept = np.full(keep, -1, np.int64)
    if n <= keep:
        kept[:n] = np.arange(n)
        return kept
    safe = (pos[:n] < first) | (pos[:n] >= seq_len - recent)
    m = mass[:n].astype(np.float64)
    # protected ones, then by mass, then what is no number; ties: the lower place
    order = sorted(range(n), key=lambda p: (not safe[p], np.isnan(m[p]) and not safe[p], 0.0 if safe[p] or np.isnan(m[p]) else -m[p], p))
    stay = np.zeros(n, bool)
    stay[order[:keep]] = True
    kept[:] = np.arange(keep)
    kept[np.flatnonzero(~stay[:keep])] = keep + np.flatnonzero(stay[keep:])
    return kept
