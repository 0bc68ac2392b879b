"""float64 statements of the key/value cache in 4 bits: format, attention over it, what its rows collect, eviction.

Arrays are NumPy.  A cache half is (codes [B, heads, capacity, dh/2] uint8, scales [B, heads, capacity, dh/32] uint8); two
codes per byte, the even channel in the low nibble; a code is a sign bit and a rank on LEVELS; scale byte t stands for
2^(t - 127), 255 for NaN.
"""
from __future__ import annotations

from typing import Optional, Sequence, Tuple

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GROUP = 32
E_MIN, E_MAX = -124, 125


def quantise(x: np.ndarray) -> Tuple[np.ndarray, np.ndarray]:
    """Codes [..., dh/2] and scale bytes [..., dh/32] of rows [..., dh]."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], 0.0, g)
    a = np.abs(g).max(-1)
    # the smallest e in range with a <= 6 2^e, looked for one by one from below
    e = np.full(a.shape, E_MIN)
    with np.errstate(divide="ignore"):
        start = np.where(a > 0, np.floor(np.log2(np.where(a > 0, a, 1.0) / 6.0)) - 1, E_MIN)
    e = np.maximum(e, start.astype(np.int64))
    for _ in range(4):
        e = np.where((a > 6.0 * np.exp2(e.astype(np.float64))) & (e < E_MAX), e + 1, e)
    e = np.minimum(e, E_MAX)
    y = np.abs(g) / np.exp2(e.astype(np.float64))[..., None]
    gap = np.abs(y[..., None] - LEVELS)                         # nearest level, the even rank of two as near
    best = gap.min(-1, keepdims=True)
    rank = np.where(gap == best, np.arange(8), 99)
    even = np.where(rank % 2 == 0, rank, 99).min(-1)
    rank = np.where(even < 99, even, rank.min(-1))
    code = (rank | (np.signbit(g).astype(np.int64) << 3)).reshape(x.shape)
    code = np.where(np.repeat(bad, GROUP, -1).reshape(x.shape), 0, code)
    codes = (code[..., 0::2] | code[..., 1::2] << 4).astype(np.uint8)
    return codes, np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    code = np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1)
    v = np.where(code >= 8, -1.0, 1.0) * LEVELS[code & 7]
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return v * np.repeat(s, GROUP, -1)


def attention(q: np.ndarray, K: np.ndarray, V: np.ndarray, scale: float, lens: Sequence[int], counts: Sequence[int]):
    """q [B, n, H, dh], K / V values [B, heads, capacity, dh].  Returns out, lse, and of every output the two sums its error
    bounds are made of: sum_j p_j |v_j| (per channel) and, per query and head, the largest sum_c |q_c k_jc| scale."""
    B, n, H, dh = q.shape
    G = H // K.shape[1]
    out = np.zeros((B, n, H, dh))
    weight = np.zeros((B, n, H, dh))
    lse = np.full((B, n, H), -np.inf)
    reach = np.zeros((B, n, H))
    for b in range(B):
        L, c = int(lens[b]), int(counts[b])
        if L == 0 or c == 0:
            continue
        for h in range(H):
            k, v = K[b, h // G, :L], V[b, h // G, :L]
            s = scale * (q[b, :c, h] @ k.T)
            top = s.max(-1, keepdims=True)
            p = np.exp(s - top)
            z = p.sum(-1, keepdims=True)
            p /= z
            out[b, :c, h] = p @ v
            weight[b, :c, h] = p @ np.abs(v)
            lse[b, :c, h] = (top + np.log(z))[:, 0]
            reach[b, :c, h] = abs(scale) * (np.abs(q[b, :c, h]) @ np.abs(k).T).max(-1)
    return out, lse, weight, reach


def mass(q: np.ndarray, K: np.ndarray, scale: float, lse: np.ndarray, mass_in: Optional[np.ndarray], lens: Sequence[int],
         counts: Sequence[int]) -> Tuple[np.ndarray, np.ndarray]:
    """Masses [B, capacity] and what was collected by this call alone.  A sum that is NaN adds nothing to a row's mass."""
    B, n, H, dh = q.shape
    G = H // K.shape[1]
    cap = K.shape[2]
    got = np.zeros((B, cap))
    out = np.full((B, cap), -1.0)
    for b in range(B):
        L, c = int(lens[b]), int(counts[b])
        for h in range(H):
            if L and c:
                s = scale * (q[b, :c, h] @ K[b, h // G, :L].T)
                got[b, :L] += np.exp(s - lse[b, :c, h][:, None]).sum(0)
        m0 = np.zeros(L) if mass_in is None else mass_in[b, :L]
        out[b, :L] = np.where(m0 > 0, m0, 0.0) + np.where(np.isnan(got[b, :L]), 0.0, got[b, :L])
    return out, got


def evict(half: Tuple[np.ndarray, np.ndarray], dst: Tuple[np.ndarray, np.ndarray], kept_idx: np.ndarray, counts: Sequence[int],
          lens: Sequence[int]) -> Tuple[np.ndarray, np.ndarray]:
    """dst after the rows kept_idx[b, :min(counts[b], lens[b])] of `half` moved to its front."""
    codes, scales = dst[0].copy(), dst[1].copy()
    for b in range(kept_idx.shape[0]):
        for s in range(min(int(counts[b]), int(lens[b]))):
            j = int(kept_idx[b, s])
            if 0 <= j < lens[b]:
                codes[b, :, s], scales[b, :, s] = half[0][b, :, j], half[1][b, :, j]
            else:
                codes[b, :, s], scales[b, :, s] = 0, 127
    return codes, scales


def block(x: np.ndarray, idx: np.ndarray, weights, K: np.ndarray, V: np.ndarray, heads: int, lens: Sequence[int],
          counts: Sequence[int], gelu_form: str = "erf", qk_scale=None, ada=None, cross=None):
    """The pruned block on cached rows as they read: K, V values [B, heads, capacity, dh], image b's kept tokens
    idx[b, :counts[b]] among its lens[b] rows (prior ones first, its own behind them); the variants are those of
    nova_oracle.pruned_block.  Returns y_kept [B, k, C], the keys and
    values [B, k, C] of the kept tokens before they are quantised, and the weight the rows collect [B, capacity]."""
    from . import nova_oracle as O
    x = np.asarray(x, dtype=np.float64)
    W = {n: np.asarray(a, dtype=np.float64) for n, a in weights.items() if a is not None}
    B, _, C = x.shape
    k, dh = idx.shape[1], C // heads
    y, kn, vn = (np.zeros((B, k, C)) for _ in range(3))
    got = np.zeros((B, K.shape[2]))
    act = {"erf": O.gelu, "tanh": O.gelu_tanh}[gelu_form]
    for b in range(B):
        c, L = int(counts[b]), int(lens[b])
        if c == 0:
            continue
        s1 = b1 = s2 = b2 = 0.0
        g1 = g2 = 1.0
        if ada is not None:
            b1, s1, g1, b2, s2, g2 = np.asarray(ada, dtype=np.float64)[b]
        xs = x[b, idx[b, :c]]
        qkv = (O.layer_norm(xs) * (1 + s1) + b1) @ W["w_qkv"].T + W.get("b_qkv", 0.0)
        q, kn[b, :c], vn[b, :c] = qkv[:, :C], qkv[:, C:2 * C], qkv[:, 2 * C:]
        a = np.zeros((c, C))
        for h in range(heads):
            sl = slice(h * dh, (h + 1) * dh)
            scale = 1 / np.sqrt(dh)
            qh = q[:, sl]
            if qk_scale is not None:
                qh, scale = O.unit_rows(qh), float(qk_scale[h])
                kn[b, :c, sl] = O.unit_rows(kn[b, :c, sl])
            p = O.softmax(scale * (qh @ K[b, h, :L].T))
            got[b, :L] += p.sum(0)
            a[:, sl] = p @ V[b, h, :L]
        x1 = xs + g1 * (a @ W["w_o"].T + W.get("b_o", 0.0))
        if cross is not None:
            t = {n: np.asarray(cross[n], dtype=np.float64) for n in ("w_cq", "b_cq", "w_co", "b_co", "k_text", "v_text")}
            qc = O.layer_norm(x1) @ t["w_cq"].T + t["b_cq"]
            ac = np.concatenate([O.softmax(qc[:, s] @ t["k_text"][b][:, s].T / np.sqrt(dh)) @ t["v_text"][b][:, s]
                                 for s in (slice(h * dh, (h + 1) * dh) for h in range(heads))], 1)
            x1 = x1 + ac @ t["w_co"].T + t["b_co"]
        hid = act((O.layer_norm(x1) * (1 + s2) + b2) @ W["w_fc1"].T + W.get("b_fc1", 0.0))
        y[b, :c] = x1 + g2 * (hid @ W["w_fc2"].T + W.get("b_fc2", 0.0))
    return y, kn, vn, got
