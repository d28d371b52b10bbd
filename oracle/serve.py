"""Oracle: the batched serving step (rotary positions with per-head norms, the append to a paged
cache, attention over it, sampling). Test infrastructure only (see the package docstring). Float64.

Readings adopted:

  * a rotation turns the first rot_dim columns of a head pair by pair, pair j by position * freqs[j]:
    columns (j, j + rot_dim / 2), or (2j, 2j + 1) when interleaved; the norm comes before it;
  * sequence b's row r lies in page table[b, r // page_size] at offset r % page_size; keys are stored
    [page, head, position, column], values [page, head, column, position];
  * token i of a sequence stands at row p + i (p its cache position) and sees rows 0 .. p + i, of the
    last `window` ones (0: all), of its own chunk only the tokens whose bits its mask has;
    score = cap tanh(scale q.k / cap) - slope (p + i - row); a token that sees nothing gets zeros;
  * sampling keeps a prefix of the tokens ordered by (logit descending, index ascending): the first
    k, of these the ones whose preceding mass is below top_p of the k tokens' mass, of these the
    ones with weight >= min_p (weights relative to the best token's 1), the best one always; the
    token is the first one in index order whose running kept mass exceeds u times the kept mass. A
    token more than 700 temperatures below the best (and a NaN) weighs nothing and is not counted.
"""

from __future__ import annotations

import math

import numpy as np

from .ffn import widen_bf16


def _f64(a):
    a = np.asarray(a)
    return widen_bf16(a) if a.dtype == np.uint16 else a.astype(np.float64)


def rope(x, positions, freqs, interleaved=False, mscale=1.0, norm_eps=-1.0, weight=None):
    """x [T, heads, hd], positions [T], freqs [rot / 2]."""
    x = _f64(x).copy()
    if norm_eps >= 0:
        x = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + norm_eps)
        if weight is not None:
            x = x * _f64(weight)
    freqs = np.asarray(freqs, dtype=np.float64)
    half = freqs.shape[0]
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        ang = np.asarray(positions, dtype=np.float64) * freqs[j]
        c, s = mscale * np.cos(ang)[:, None], mscale * np.sin(ang)[:, None]
        u, v = x[:, :, a].copy(), x[:, :, b].copy()
        x[:, :, a], x[:, :, b] = u * c - v * s, u * s + v * c
    return x


def places(cache_pos, tok_start, table, page_size, n_pages):
    """(token, sequence, row, page) of every token that has a place; page -1 where it is a bad one."""
    out = []
    cap = table.shape[1] * page_size
    for b, p in enumerate(np.asarray(cache_pos).tolist()):
        s, e = int(tok_start[b]), int(tok_start[b + 1])
        for t in range(s, e):
            row = p + t - s
            page = -1
            if p >= 0 and p + (e - s) <= cap:
                page = int(table[b, row // page_size])
                if page >= n_pages:
                    page = -1
            out.append((t, b, row, page))
    return out


def attn_paged(q, k_pages, v_pages, table, cache_pos, tok_start, scale=None, softcap=0.0, slopes=None, window=0,
               mask=None):
    """q [T, H, hd]; k_pages [pages, Hkv, ps, hd], v_pages [pages, Hkv, hd, ps]. Returns [T, H, hd]; rows
    of tokens of no sequence are NaN here (a caller compares the others)."""
    q = _f64(q)
    kp, vp = _f64(k_pages), _f64(v_pages)
    t_n, h, hd = q.shape
    n_pages, hkv, ps, _ = kp.shape
    scale = 1.0 / math.sqrt(hd) if scale is None else scale
    out = np.full((t_n, h, hd), np.nan)
    for b, p in enumerate(np.asarray(cache_pos).tolist()):
        s, e = int(tok_start[b]), int(tok_start[b + 1])
        length = p + e - s
        if e == s or p < 0 or length > table.shape[1] * ps:
            continue
        rows = np.arange(length)
        ids = np.asarray(table[b])[rows // ps]
        bad = (ids < 0) | (ids >= n_pages)
        ids = np.where(bad, 0, ids)
        keys, values = kp[ids, :, rows % ps], vp[ids, :, :, rows % ps]  # [length, Hkv, hd]
        for t in range(s, e):
            row = p + t - s
            seen = rows <= row
            if window > 0:
                seen &= rows > row - window
            if mask is not None:
                for j in range(e - s):
                    if not (int(mask[t]) >> j) & 1:
                        seen[p + j] = False
            if (seen & bad).any():
                continue
            for hh in range(h):
                g = hh // (h // hkv)
                if not seen.any():
                    out[t, hh] = 0.0
                    continue
                x = keys[seen, g] @ q[t, hh] * scale
                if softcap > 0:
                    x = softcap * np.tanh(x / softcap)
                if slopes is not None:
                    x = x - float(slopes[hh]) * (row - rows[seen])
                w = np.exp(x - x.max())
                out[t, hh] = (w / w.sum()) @ values[seen, g]
    return out


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row. Returns (token, kept, probability of the token among the kept)."""
    x = np.asarray(logits, dtype=np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    best = x.max()
    if best == -np.inf:
        return -1, 0, 0.0
    if temperature == 0:
        return int(np.argmax(x)), 1, 1.0
    with np.errstate(invalid="ignore"):
        z = (x - best) / temperature
        w = np.where(z >= -700.0, np.exp(z), 0.0) if np.isfinite(best) else (x == best).astype(np.float64)
    order = np.argsort(-x, kind="stable")
    order = order[w[order] > 0]  # what weighs nothing is never drawn and not counted
    if top_k > 0:
        order = order[:top_k]
    if top_p < 1:
        ahead = np.concatenate(([0.0], np.cumsum(w[order])[:-1]))
        order = order[: max(1, int(np.sum(ahead < top_p * w[order].sum())))]
    order = order[: max(1, int(np.sum(w[order] >= min_p)))]
    kept = np.sort(order)
    run = np.cumsum(w[kept])
    j = min(int(np.sum(run <= u * run[-1])), len(kept) - 1)
    return int(kept[j]), len(kept), float(w[kept[j]] / run[-1])
