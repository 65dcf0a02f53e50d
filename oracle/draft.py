"""Oracle of decoding with drafted tokens: plain loops over requests, rows and tokens, values in 64 bits.

Arrays come decoded (float64 / int); pages as the library keeps them: K [pages][heads][page][dim],
V [pages][heads][page / e][dim][e].
"""
from __future__ import annotations

from typing import List, Sequence, Tuple

import numpy as np


def sees(tree, t: int, node: int, n: int) -> List[int]:
    """Nodes of its own request that row t sees (tree: words, or None for a chain)."""
    word = ((1 << (node + 1)) - 1) if tree is None else int(tree[t]) & (1 << 64) - 1
    return [j for j in range(n) if (word >> j) & 1]


def parent(tree, t: int, node: int) -> int:
    up = [j for j in sees(tree, t, node, node)]
    return up[-1] if up else -1


def cached(K: np.ndarray, V: np.ndarray, ids: Sequence[int], length: int, head: int) -> Tuple[np.ndarray, np.ndarray]:
    """K and V [tokens][dim] of one request and head; tokens in pages that do not exist are left out."""
    pages, _, page, dim = K.shape
    e = V.shape[4]
    k, v = [], []
    for j in range(length):
        p, at = ids[j // page], j % page
        if 0 <= p < pages:
            k.append(K[p, head, at])
            v.append(V[p, head, at // e, :, at % e])
    return np.array(k).reshape(-1, dim), np.array(v).reshape(-1, dim)


def attention(K, V, q, k, v, tree, table, lens, starts, scale: float, max_nodes: int = 64):
    """(out, lse, weight, reach) of the rows of requests: out [T][heads_q][dim], lse [T][heads_q]; weight = sum of p |v| and
    reach = the largest scale * sum |q| |k| over the tokens a row sees, which rounding errors scale with.  Rows that belong to no request: NaN."""
    T, hq, dim = q.shape
    heads = k.shape[1]
    out = np.full((T, hq, dim), np.nan)
    lse = np.full((T, hq), np.nan)
    weight = np.full((T, hq, dim), np.nan)
    reach = np.zeros((T, hq))
    for r, length in enumerate(lens):
        a, n = int(starts[r]), min(int(starts[r + 1]) - int(starts[r]), max_nodes)
        for h in range(heads):
            kc, vc = cached(K, V, table[r], int(length), h)
            for i in range(n):
                s = sees(tree, a + i, i, n)
                kk = np.concatenate([kc, k[a:a + n, h][s]])
                vv = np.concatenate([vc, v[a:a + n, h][s]])
                for g in range(h * (hq // heads), (h + 1) * (hq // heads)):
                    z = scale * (kk @ q[a + i, g])
                    top = z.max() if z.size else -np.inf
                    p = np.exp(z - top) if top > -np.inf else np.zeros(z.size)
                    total = p.sum()
                    p = p / total if total > 0 else p
                    out[a + i, g] = p @ vv
                    weight[a + i, g] = p @ np.abs(vv)
                    lse[a + i, g] = top + np.log(total) if total > 0 else -np.inf
                    reach[a + i, g] = abs(scale) * (np.abs(kk) @ np.abs(q[a + i, g])).max() if z.size else 0.0
    return out, lse, weight, reach


def best_token(row: np.ndarray) -> int:
    """Lowest index of the largest value, NaN above all."""
    nan = np.flatnonzero(np.isnan(row))
    return int(nan[0]) if nan.size else int(np.flatnonzero(row == row.max())[0])


def accept(logits, tokens, tree, starts):
    """(keep [T], counts [R], next [R], best [T])."""
    T = len(logits)
    best = [best_token(row) for row in logits]
    keep, counts, following = [-1] * T, [], []
    for r in range(len(starts) - 1):
        a, n = int(starts[r]), int(starts[r + 1]) - int(starts[r])
        if n == 0:
            counts.append(0)
            following.append(-1)
            continue
        at, count = 0, 1
        keep[a] = 0
        while True:
            fit = [j for j in range(at + 1, n) if parent(tree, a + j, j) == at and tokens[a + j] == best[a + at]]
            if not fit:
                break
            at = fit[0]
            keep[a + at] = count
            count += 1
        counts.append(count)
        following.append(best[a + at])
    return keep, counts, following, best


def plan(table, ring, pool, lens, add, starts, page: int, keep, rows: int):
    """(slots, lens, pool, refused, table, ring) after the step; the arguments stay as they are."""
    table, ring = [list(r) for r in table], list(ring)
    old, before_ring = [list(r) for r in table], list(ring)
    pages, width = len(ring), len(table[0])
    head, free = pool
    up = lambda n: -(-n // page)
    taken, want, back = 0, 0, []
    lens_out, refused, extra = [], [], []
    for r, (n, a) in enumerate(zip(lens, add)):
        if a < 0:
            back += old[r][:up(n)]
            lens_out.append(0)
            refused.append(0)
            extra.append(0)
            continue
        need = up(n + a) - up(n)
        no = up(n + a) > width
        if not no and need > 0:
            want += need
            no = want > free
        if no:
            lens_out.append(n)
            refused.append(1)
            extra.append(0)
            continue
        for i in range(need):
            table[r][up(n) + i] = before_ring[(head + want - need + i) % pages]
        taken = want if need else taken
        lens_out.append(n + a)
        refused.append(0)
        extra.append(a)
    for i, p in enumerate(back):
        ring[(head + free + i) % pages] = p
    slots = [-1] * rows
    for r in range(len(lens)):
        for t in range(int(starts[r]), min(int(starts[r + 1]), rows)):
            place = t - int(starts[r]) if keep is None else keep[t]
            if 0 <= place < extra[r]:
                at = lens[r] + place
                slots[t] = table[r][at // page] * page + at % page
    return slots, lens_out, [(head + taken) % pages, free - taken + len(back)], refused, table, ring


def commit(K: np.ndarray, V: np.ndarray, k: np.ndarray, v: np.ndarray, slots) -> None:
    """K [layers][pages][heads][page][dim] and V [layers][pages][heads][page / e][dim][e] in place."""
    pages, page, e = K.shape[1], K.shape[3], V.shape[5]
    for t, s in enumerate(slots):
        if 0 <= s < pages * page:
            K[:, s // page, :, s % page] = k[:, t]
            V[:, s // page, :, s % page // e, :, s % e] = v[:, t]
