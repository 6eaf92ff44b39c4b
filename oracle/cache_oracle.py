"""The definitions behind a bounded cache in 64 bits: attention with changed scores, attention weights of cache rows, eviction.

TEST INFRASTRUCTURE like s4c_oracle.py: plain numpy, a row at a time, no code of the library.  Arrays are float64 unless they are
whole numbers; caches are [B][Hkv][S_cap][D] (gather_pages makes one of a paged pool).
"""
from __future__ import annotations

import numpy as np


def gather_pages(pool, table):
    """pool [pages][Hkv][page][D], table [B][blocks] -> [B][Hkv][blocks * page][D]"""
    B, blocks = table.shape
    _, Hkv, page, D = pool.shape
    return pool[table].transpose(0, 2, 1, 3, 4).reshape(B, Hkv, blocks * page, D)


def changed(x, cap, slope, distance):
    """scores x of one query head (scaled already); distance: the keys' positions from the root's"""
    if cap > 0:
        x = cap * np.tanh(x / cap)
    return x if slope is None else x + slope * distance


def ancestors_or_self(parent):
    rows = []
    for i in range(len(parent)):
        row, j = [], i
        while j >= 0:
            row.append(j)
            j = parent[j]
        rows.append(row[::-1])
    return rows


def tree_attn_scored(q, k_tree, v_tree, k_cache, v_cache, cache_len, parent, scale=0.0, cap=0.0, slopes=None, key_pos=None, root_pos=None):
    """out [B][N][Hq][D], lse [B][N][Hq], and for tolerances, p the softmax and s = |capped score| + |bias| of every key: sums of p |v| and of
    p s |v| [B][N][Hq][D], of p s [B][N][Hq], and the largest sum |q k| scale of a row [B][N][Hq]"""
    B, N, Hq, D = q.shape
    Hkv = k_tree.shape[2]
    scale = scale if scale > 0 else 1.0 / np.sqrt(D)
    out, mean, mean_s = (np.zeros((B, N, Hq, D)) for _ in range(3))
    lse, size, mass = (np.zeros((B, N, Hq)) for _ in range(3))
    for b in range(B):
        n = cache_len[b]
        for h in range(Hq):
            g = h // (Hq // Hkv)
            dist = np.arange(n) - n if key_pos is None else key_pos[b, g, :n].astype(np.int64) - int(root_pos[b])
            for i, seen in enumerate(ancestors_or_self(parent[b])):
                k = np.concatenate([k_cache[b, g, :n], k_tree[b, seen, g]])
                v = np.concatenate([v_cache[b, g, :n], v_tree[b, seen, g]])
                d = np.concatenate([dist, np.arange(len(seen))])
                x = changed(k @ q[b, i, h] * scale, cap, None if slopes is None else slopes[h], d)
                m = x.max()
                p = np.exp(x - m)
                lse[b, i, h] = m + np.log(p.sum())
                p /= p.sum()
                bias = 0.0 if slopes is None else slopes[h] * d
                s = np.abs(x - bias) + np.abs(bias)
                out[b, i, h], mean[b, i, h], mean_s[b, i, h] = p @ v, p @ np.abs(v), (p * s) @ np.abs(v)
                size[b, i, h] = p @ s
                mass[b, i, h] = (np.abs(k) @ np.abs(q[b, i, h])).max() * scale
    return out, lse, mean, mean_s, size, mass


def kv_weigh(q, k_cache, lse, cache_len, path, accept_len, weight_in, scale=0.0, cap=0.0, slopes=None, key_pos=None, root_pos=None):
    """weight and key_pos after (copies), and the part of `weight` that this call added"""
    B, _, Hq, D = q.shape
    Hkv = k_cache.shape[1]
    scale = scale if scale > 0 else 1.0 / np.sqrt(D)
    weight, added = weight_in.copy(), np.zeros_like(weight_in)
    pos = None if key_pos is None else key_pos.copy()
    for b in range(B):
        n, L = int(cache_len[b]), int(accept_len[b])
        first = n - (L + 1)
        for g in range(Hkv):
            dist = np.arange(n) - first
            if pos is not None:
                pos[b, g, first:n] = root_pos[b] + np.arange(L + 1)
                dist = pos[b, g, :n].astype(np.int64) - int(root_pos[b])
            weight[b, g, first:n] = 0.0
            for k in range(L + 1):
                m = first + k + 1
                for h in range(g * (Hq // Hkv), (g + 1) * (Hq // Hkv)):
                    x = changed(k_cache[b, g, :m] @ q[b, path[b, k], h] * scale, cap, None if slopes is None else slopes[h], dist[:m])
                    added[b, g, :m] += np.exp(x - lse[b, path[b, k], h])
            weight[b, g, :n] += added[b, g, :n]
    return weight, pos, added


def kv_evict(weight, key_pos, cache_len, next_pos, budget, recent):
    """kept [layers][B][Hkv][budget]: the row that row i was before, -1 behind the new length; new_len [B]"""
    layers, B, Hkv, _ = weight.shape
    kept = np.full((layers, B, Hkv, budget), -1, dtype=np.int32)
    new_len = np.minimum(cache_len, budget)
    for ly, b, g in np.ndindex(layers, B, Hkv):
        n, m = int(cache_len[b]), int(new_len[b])
        rows = range(n)
        if n > budget:
            rank = sorted(rows, key=lambda j: (key_pos[ly, b, g, j] < int(next_pos[b]) - recent, -weight[ly, b, g, j] if
                                               key_pos[ly, b, g, j] < int(next_pos[b]) - recent else 0.0, j))
            stays = set(rank[:m])
        else:
            stays = set(rows)
        movers = iter(sorted(j for j in stays if j >= m))
        kept[ly, b, g, :m] = [j if j in stays else next(movers) for j in range(m)]
        assert next(movers, None) is None
    return kept, new_len
