"""Reference oracle of a key/value cache in pages -- TEST INFRASTRUCTURE ONLY:
plain float64 numpy definitions, nothing shared with the product.

Pools are [pages, heads, places of a page, D]; row b of `table` names the pages
of sequence b; its new tokens are rows first[b] .. first[b + 1] - 1 of packed
tensors and the last of its lens[b] places.
"""
from __future__ import annotations

import numpy as np


def tokens(table, first, lens, page):
    """(row, sequence, place) of every new token."""
    cap = table.shape[1] * page
    for b in range(len(lens)):
        n = int(first[b + 1] - first[b])
        for i in range(n):
            yield int(first[b]) + i, b, int(lens[b]) - n + i, cap


def rotate(x, place, turns, layout, amplitude=1.0):
    """x [heads, D] with its first 2 len(turns) channels rotated for a token at a place."""
    y = x.copy()
    n = len(turns)
    for i in range(n):
        a = 2 * np.pi * ((place * turns[i]) % 1.0)
        i0, i1 = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, n + i)
        y[:, i0] = amplitude * (x[:, i0] * np.cos(a) - x[:, i1] * np.sin(a))
        y[:, i1] = amplitude * (x[:, i0] * np.sin(a) + x[:, i1] * np.cos(a))
    return y


def norm(x, w, eps):
    return x if w is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w


def append(q, k, v, pool_k, pool_v, table, first, lens, w_q=None, w_k=None, eps=1e-6, turns=(), layout="half",
           amplitude=1.0):
    """q as it comes out (unrounded), the pools with the new tokens' unrounded keys and values, and which places were
    written (bool [pages, places])."""
    pool_k, pool_v = pool_k.copy(), pool_v.copy()
    out = None if q is None else q.copy()
    page = pool_k.shape[2]
    written = np.zeros((pool_k.shape[0], page), bool)
    for t, b, p, cap in tokens(table, first, lens, page):
        if q is not None:
            out[t] = rotate(norm(q[t], w_q, eps), p, turns, layout, amplitude)
        if not 0 <= p < cap:
            continue
        at = int(table[b, p // page])
        if not 0 <= at < pool_k.shape[0]:
            continue
        pool_k[at, :, p % page] = rotate(norm(k[t], w_k, eps), p, turns, layout, amplitude)
        pool_v[at, :, p % page] = v[t]
        written[at, p % page] = True
    return out, pool_k, pool_v, written


def means(pool_k, table, first, lens, old):
    """Mean keys: of each page that new tokens touch over its places below lens[b] (from pool_k, as stored); `old` elsewhere."""
    out, page = old.copy(), pool_k.shape[2]
    for _, b, p, cap in tokens(table, first, lens, page):
        if not 0 <= p < cap:
            continue
        at = int(table[b, p // page])
        if 0 <= at < pool_k.shape[0]:
            n = min(page, int(lens[b]) - p // page * page)
            out[at] = pool_k[at, :, :n].mean(1)
    return out


def gather(pool, table, b, h, places):
    """Rows of the places that lie on pages of the pool, and which of the places those are."""
    page = pool.shape[2]
    at = table[b, places // page]
    there = (at >= 0) & (at < pool.shape[0])
    return pool[at[there], h, places[there] % page], there


def attn(q, pool_k, pool_v, table, first, lens, causal, scale, selected=None, q_block=1):
    """O [T, H, D], LSE [H, T], sum of weight |v| and sum over d of |q||k| at most over a row's keys (for error bounds); rows
    of no sequence: NaN."""
    T, H, D = q.shape
    heads, page = pool_k.shape[1:3]
    G, cap = H // heads, table.shape[1] * page
    o, mag = np.full(q.shape, np.nan), np.zeros(q.shape)
    lse, big = np.full((H, T), np.nan), np.zeros((H, T))
    for b in range(len(lens)):
        f0, f1 = int(first[b]), int(first[b + 1])
        n = min(max(int(lens[b]), 0), cap)
        for t in range(f0, f1):
            see = n - f1 + t + 1 if causal else n
            for hk in range(heads):
                if selected is None:
                    places = np.arange(max(see, 0))
                else:
                    s = selected[f0 // q_block + b + (t - f0) // q_block, hk]
                    s = s[(s >= 0) & (s < table.shape[1])].astype(np.int64)
                    places = (s[:, None] * page + np.arange(page)).reshape(-1)
                    places = places[places < see]
                k, there = gather(pool_k, table, b, hk, places)
                v, _ = gather(pool_v, table, b, hk, places)
                for h in range(hk * G, (hk + 1) * G):
                    if len(k) == 0:
                        o[t, h], lse[h, t] = 0.0, -np.inf
                        continue
                    s = k @ q[t, h] * scale
                    p = np.exp(s - s.max())
                    o[t, h], mag[t, h] = p @ v / p.sum(), p @ np.abs(v) / p.sum()
                    lse[h, t] = s.max() + np.log(p.sum())
                    big[h, t] = (np.abs(k) @ np.abs(q[t, h])).max() * scale
    return o, lse, mag, big


def select(q, means, table, first, lens, page, count, q_block, keep_first, keep_last, causal):
    """int32 [T // q_block + B, heads, count]: pages ascending, -1 behind the last."""
    T, H, D = q.shape
    heads, B = means.shape[1], len(lens)
    out = np.full((T // q_block + B, heads, count), -1, np.int32)
    for b in range(B):
        f0, f1 = int(first[b]), int(first[b + 1])
        n = min(max(int(lens[b]), 0), table.shape[1] * page)
        for j, t in enumerate(range(f0, f1, q_block)):
            end = min(t + q_block, f1)
            see = max(n - f1 + end, 0) if causal else n
            pages = -(-see // page)
            for hk in range(heads):
                x = q[t:end, hk * (H // heads):(hk + 1) * (H // heads)].sum((0, 1))
                at = table[b, :pages]
                there = (at >= 0) & (at < means.shape[0])
                with np.errstate(invalid="ignore"):
                    score = np.where(there, means[np.where(there, at, 0), hk] @ x, -np.inf)
                score = np.where(np.isnan(score), -np.inf, score)
                must = [p for p in range(pages) if p < keep_first or p >= pages - keep_last]
                rest = sorted((p for p in range(pages) if p not in must), key=lambda p: (-score[p], p))
                picks = sorted(must + rest[:max(0, count - len(must))])[:count] if pages > count else list(range(pages))
                out[f0 // q_block + b + j, hk, :len(picks)] = picks
    return out
