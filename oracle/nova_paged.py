"""float64 statements of the key/value cache in pages: page lists, slots, attention over it, means of pages, which pages a query reads.

Arrays are NumPy.  A pool half is [pages, kv_heads, page_rows, dh]; row r of image b lies in page table[b, r // page_rows], row
r % page_rows of it, and is zeros where that entry is no page.
"""
from __future__ import annotations

from typing import List, Optional, Sequence, Tuple

import numpy as np


def reserve(table: np.ndarray, page_rows: int, free_pages: Sequence[int], free_count: int, now: Sequence[int], keep: Sequence[int],
            come: Sequence[int], n: int):
    """table, slots [B, n], rows of the images afterwards, free_pages and its height, one page after the other."""
    B, pages = len(now), len(free_pages)
    table = table.copy()
    stack = list(free_pages[:min(max(free_count, 0), pages)])
    pages_of = lambda rows: -(-rows // page_rows)
    for b in range(B):
        for i in range(pages_of(keep[b] + come[b]), pages_of(now[b])):
            stack.append(int(table[b, i]))
    after, slots, empty = [], np.full((B, n), -1, dtype=np.int64), False
    for b in range(B):
        held, rows = pages_of(now[b]), keep[b] + come[b]
        grows = pages_of(rows) - held
        if grows > 0:
            empty = empty or grows > len(stack)
            if empty:
                rows = min(rows, held * page_rows)
            else:
                for i in range(grows):
                    table[b, held + i] = stack.pop()
        after.append(rows)
        for r in range(keep[b], rows):
            page = int(table[b, r // page_rows])
            if 0 <= page < pages:
                slots[b, r - keep[b]] = page * page_rows + r % page_rows
    out = np.array(free_pages, dtype=np.int64)
    height = min(len(stack), pages)
    out[:height] = stack[:height]
    return table, slots, after, out, height


def append(pool: np.ndarray, rows: np.ndarray, slots: np.ndarray) -> np.ndarray:
    """The pool half after rows [B, n, kv_heads, dh] went to their slots."""
    pool = pool.copy()
    p = pool.shape[2]
    for b, s in np.argwhere((slots >= 0) & (slots < pool.shape[0] * p)):
        pool[slots[b, s] // p, :, slots[b, s] % p] = rows[b, s]
    return pool


def image_rows(pool: np.ndarray, table_row: np.ndarray, length: int) -> np.ndarray:
    """[kv_heads, length, dh]: an image's rows, one after the other."""
    pages, hk, p, dh = pool.shape
    out = np.zeros((hk, length, dh))
    for i in range(-(-length // p)):
        m = min(p, length - i * p)
        if 0 <= table_row[i] < pages:
            out[:, i * p:i * p + m] = pool[table_row[i], :, :m]
    return out


def visible(length: int, count: int, n: int, causal: bool) -> np.ndarray:
    """Rows that each of n queries sees, the first `count` of them live."""
    s = np.arange(n)
    v = np.clip(length - count + s + 1, 0, length) if causal else np.full(n, length)
    return np.where(s < count, v, 0)


def attention(q: np.ndarray, K: List[np.ndarray], V: List[np.ndarray], scale: float, counts: Sequence[int], causal: bool,
              chosen: Optional[np.ndarray] = None, page_rows: int = 0):
    """q [B, n, H, dh]; K, V per image [kv_heads, length, dh]; chosen [B, n, kv_heads, k] or None.  Returns out, lse, and what error
    bounds are made of: sum_j p_j |v_j| per channel and the largest sum_c |q_c k_jc| scale.  Rows that a query does not see have
    no part in anything."""
    B, n, H, dh = q.shape
    out, weight = np.zeros((B, n, H, dh)), np.zeros((B, n, H, dh))
    lse, reach = np.full((B, n, H), -np.inf), np.zeros((B, n, H))
    for b in range(B):
        hk, L, _ = K[b].shape
        G = H // hk
        vis = visible(L, int(counts[b]), n, causal)
        for h in range(H):
            k, v = K[b][h // G], V[b][h // G]
            for s in range(n):
                see = np.arange(L) < vis[s]
                if chosen is not None:
                    pages = np.unique(chosen[b, s, h // G])
                    see &= np.isin(np.arange(L) // page_rows, pages[pages >= 0])
                if not see.any():
                    continue
                ks, vs = k[see], v[see]
                with np.errstate(invalid="ignore", over="ignore"):
                    t = scale * (ks @ q[b, s, h])
                    p = np.exp(t - t.max())
                    z = p.sum()
                    p /= z
                    out[b, s, h] = p @ vs
                    weight[b, s, h] = p @ np.abs(vs)
                    lse[b, s, h] = t.max() + np.log(z)
                    reach[b, s, h] = abs(scale) * (np.abs(ks) @ np.abs(q[b, s, h])).max()
    return out, lse, weight, reach


def seven_bits(x: np.ndarray) -> np.ndarray:
    """All of x as the nearest multiples w 2^e of one power of two, the smallest with |x| <= 127 2^e everywhere,
    -100 <= e <= 100."""
    if not np.isfinite(x).all():
        return np.full_like(x, np.nan)
    e = -100
    while np.abs(x).max() > 127 * 2.0 ** e and e < 100:
        e += 1
    return np.clip(np.rint(x / 2.0 ** e), -127, 127) * 2.0 ** e


def summarise(pool: np.ndarray, table: np.ndarray, means: np.ndarray, lens: Sequence[int], counts: Sequence[int]) -> np.ndarray:
    """means [pages, kv_heads, dh] after those of the pages of the images' last counts[b] rows were taken anew."""
    pages, hk, p, dh = pool.shape
    means = means.copy()
    for b, L in enumerate(lens):
        first = max(L - counts[b], 0)
        if first >= L:
            continue
        for i in range(first // p, -(-L // p)):
            page = table[b, i]
            if 0 <= page < pages:
                m = min(p, L - i * p)
                for j in range(hk):
                    means[page, j] = seven_bits(pool[page, j, :m].sum(0) / m)
    return means


def select(q: np.ndarray, means: np.ndarray, table: np.ndarray, page_rows: int, lens: Sequence[int], counts: Sequence[int], causal: bool,
           first: int, recent: int, k: int) -> np.ndarray:
    """chosen [B, n, kv_heads, k]: the `first` and `recent` pages in any case, then pages with a mean of NaN, then by score; of two
    alike the lower."""
    B, n, H, dh = q.shape
    pages, hk, _ = means.shape
    G = H // hk
    chosen = np.full((B, n, hk, k), -1, dtype=np.int64)
    for b in range(B):
        vis = visible(int(lens[b]), int(counts[b]), n, causal)
        for s in range(n):
            P = -(-int(vis[s]) // page_rows)
            if P == 0:
                continue
            ids = table[b, :P]
            for j in range(hk):
                m = np.where(((ids >= 0) & (ids < pages))[:, None], means[np.clip(ids, 0, pages - 1), j], 0.0)
                w = seven_bits(q[b, s, j * G:(j + 1) * G])
                score = (np.where(np.isnan(w), 0.0, w) @ m.T).max(0)
                rank = np.where(np.isnan(m).any(1), 1, 2)
                rank[:first] = 0
                rank[max(P - recent, 0):] = 0
                best = sorted(range(P), key=lambda i: (rank[i], -score[i] if rank[i] == 2 else 0.0, i))[:k]
                chosen[b, s, j, :len(best)] = sorted(best)
    return chosen
