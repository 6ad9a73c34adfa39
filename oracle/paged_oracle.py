"""float64 oracle of the paged-cache calls, written from their definitions (numpy, loops where loops are plainest).

A cache is k, v [n_pages, n_kv_heads, page_size, head_dim] with an int page table [batch, max_pages]; position t of
sequence b is slot t % page_size of page table[b, t // page_size].  A sequence's new tokens are its last positions.
"""
from __future__ import annotations

import numpy as np


def rows(x, table_row, n):
    """Rows 0 .. n-1 of a sequence, [n_kv_heads, n, head_dim]."""
    ps = x.shape[2]
    out = np.empty((x.shape[1], n, x.shape[3]))
    for t in range(n):
        out[:, t] = x[table_row[t // ps], :, t % ps]
    return out


def rotate(x, position, inv_freq, pairs):
    """x [heads, head_dim] of the token at `position`."""
    y = x.astype(np.float64).copy()
    half = 0 if inv_freq is None else len(inv_freq)
    for i in range(half):
        w = float(position) * float(inv_freq[i])
        a, c = (2 * i, 2 * i + 1) if pairs else (i, i + half)
        y[:, a] = x[:, a] * np.cos(w) - x[:, c] * np.sin(w)
        y[:, c] = x[:, c] * np.cos(w) + x[:, a] * np.sin(w)
    return y


def append(k, v, table, kv_lens, cu_q, k_new, v_new, inv_freq=None, pairs=False, positions=None):
    """Caches with the new rows (new arrays; not rounded)."""
    k, v, ps = k.copy(), v.copy(), k.shape[2]
    for b in range(len(kv_lens)):
        q = cu_q[b + 1] - cu_q[b]
        for i in range(q):
            t, tok = kv_lens[b] - q + i, cu_q[b] + i
            k[table[b, t // ps], :, t % ps] = rotate(k_new[tok], t if positions is None else positions[tok], inv_freq, pairs)
            v[table[b, t // ps], :, t % ps] = v_new[tok]
    return k, v


def page_bounds(k, table, kv_lens):
    """{physical page: (min, max) [n_kv_heads, head_dim] over its rows below the sequence's length}."""
    ps, out = k.shape[2], {}
    for b, n in enumerate(kv_lens):
        for p in range((n + ps - 1) // ps):
            have = k[table[b, p], :, :min(ps, n - p * ps)]
            out[int(table[b, p])] = (have.min(1), have.max(1))
    return out


def attend(q, keys, values, visible, scale):
    """One query vector over the rows with visible[t]: (y, lse, sum p |v| / sum p)."""
    if not visible.any():
        return np.zeros(values.shape[1]), -np.inf, np.zeros(values.shape[1])
    s = keys[visible] @ q * scale
    m = s.max()
    p = np.exp(s - m)
    return p @ values[visible] / p.sum(), m + np.log(p.sum()), p @ np.abs(values[visible]) / p.sum()


def attention(q, k, v, table, kv_lens, cu_q, causal=True, scale=None):
    """q [total_q, n_q_heads, head_dim]: (y, lse, A, C), A = sum p |v| / sum p, C = max_t sum_c |q_c k_tc| * scale (what
    rounding errors of the two products scale with)."""
    T, hq, d = q.shape
    G = hq // k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    y, A = np.zeros((T, hq, d)), np.zeros((T, hq, d))
    lse, C = np.full((T, hq), -np.inf), np.zeros((T, hq))
    for b in range(len(kv_lens)):
        n, m = int(kv_lens[b]), int(cu_q[b + 1] - cu_q[b])
        if m == 0:
            continue
        K, V = rows(k, table[b], n), rows(v, table[b], n)
        for i in range(m):
            visible = np.arange(n) <= (n - m + i if causal else n - 1)
            for h in range(hq):
                t = cu_q[b] + i
                y[t, h], lse[t, h], A[t, h] = attend(q[t, h], K[h // G], V[h // G], visible, scale)
                if visible.any():
                    C[t, h] = (np.abs(K[h // G][visible]) @ np.abs(q[t, h])).max() * scale
    return y, lse, A, C


def select_pages(q_group, lo, hi, n_seen, sink, tail, topk):
    """Pages that one token's group of queries [G, head_dim] takes; lo, hi [n_seen, head_dim]."""
    bound = np.maximum(q_group[:, None] * lo, q_group[:, None] * hi).sum(2).max(0)
    forced = [p for p in range(n_seen) if p < sink or p >= n_seen - tail]
    middle = [p for p in range(n_seen) if sink <= p < n_seen - tail]
    best = sorted(middle, key=lambda p: (-bound[p], p))[:topk]
    return sorted(set(forced) | set(best))


def block_attention(q, k, v, table, kv_lens, cu_q, bounds, sink, tail, topk, scale=None):
    """(y, lse, A, C, pages [total_q, n_kv_heads, sink + tail + topk] padded with -1); bounds [n_pages, heads, 2, d]."""
    T, hq, d = q.shape
    hkv, ps = k.shape[1], k.shape[2]
    G = hq // hkv
    scale = d ** -0.5 if scale is None else scale
    y, A = np.zeros((T, hq, d)), np.zeros((T, hq, d))
    lse, C = np.full((T, hq), -np.inf), np.zeros((T, hq))
    pages = np.full((T, hkv, sink + tail + topk), -1, np.int64)
    for b in range(len(kv_lens)):
        n, m = int(kv_lens[b]), int(cu_q[b + 1] - cu_q[b])
        if m == 0:
            continue
        K, V = rows(k, table[b], n), rows(v, table[b], n)
        for i in range(m):
            t, pos = cu_q[b] + i, n - m + i
            seen = pos // ps + 1
            for h in range(hkv):
                take = select_pages(q[t, h * G:(h + 1) * G], bounds[table[b, :seen], h, 0], bounds[table[b, :seen], h, 1],
                                    seen, sink, tail, topk)
                pages[t, h, :len(take)] = take
                visible = np.isin(np.arange(n) // ps, take) & (np.arange(n) <= pos)
                for g in range(h * G, (h + 1) * G):
                    y[t, g], lse[t, g], A[t, g] = attend(q[t, g], K[h], V[h], visible, scale)
                    C[t, g] = (np.abs(K[h][visible]) @ np.abs(q[t, g])).max() * scale
    return y, lse, A, C, pages
