"""Trees of drafted tokens, chosen pages and eviction over a paged key/value
cache (include/dex.h), from their definitions in float64 and one thing at a
time: the library's kernels are tested against these."""
from __future__ import annotations

import math

import numpy as np

from .paged import page_of


def ancestors(parent, i):
    """Node i and the nodes it follows, the nearest first."""
    out = [i]
    while 0 <= parent[out[-1]] < out[-1]:
        out.append(int(parent[out[-1]]))
    return out


def tree_mask(parent):
    """(seen [n, t, t] bool, depth [n, t])."""
    n, t = parent.shape
    seen, depth = np.zeros((n, t, t), bool), np.zeros((n, t), np.int32)
    for b in range(n):
        for i in range(t):
            up = ancestors(parent[b], i)
            seen[b, i, up] = True
            depth[b, i] = len(up) - 1
    return seen, depth


def words(seen):
    """The bits of [..., t] as int64 words [..., ceil(t / 64)]."""
    t = seen.shape[-1]
    n = -(-t // 64)
    out = np.zeros(seen.shape[:-1] + (n,), np.uint64)
    for j in range(t):
        out[..., j // 64] |= seen[..., j].astype(np.uint64) << np.uint64(j % 64)
    return out.view(np.int64)


def tree_accept(parent, token, target, n_draft=None, root=None):
    n, t = parent.shape
    path, count, following = np.full((n, t), -1, np.int32), np.zeros(n, np.int32), np.zeros(n, np.int32)
    for b in range(n):
        d = t if n_draft is None else max(0, min(t, int(n_draft[b])))
        best = []
        for i in range(d):
            up = ancestors(parent[b], i)[::-1]
            ok = root is None or token[b, up[0]] == root[b]
            ok = ok and all(token[b, j] == target[b, p] for p, j in zip(up, up[1:]))
            if ok and len(up) > len(best):
                best = up
        path[b, :len(best)], count[b] = best, len(best)
        following[b] = target[b, best[-1]] if best else -1 if root is None else root[b]
    return path, count, following


def attend(q, k_pages, v_pages, places, scale=None):
    """q [rows, heads, hd]; places(r, g) lists what row r's heads of kv head g see,
    as (page, slot).  (out, lse, spread, size) as `paged.attention` has them, and
    the weights [r][g] summed over the heads."""
    rows, heads, hd = q.shape
    kv = k_pages.shape[1]
    scale = hd ** -0.5 if scale is None else scale
    out, lse, spread = np.zeros(q.shape), np.full((rows, heads), -np.inf), np.zeros(q.shape)
    size = np.zeros((rows, heads))
    weights = [[None] * kv for _ in range(rows)]
    for r in range(rows):
        for g in range(kv):
            at = places(r, g)
            weights[r][g] = np.zeros(len(at))
            if not at:
                continue
            page, slot = np.array(at).T
            k, v = k_pages[page, g, slot], v_pages[page, g, slot]
            for h in range(g * heads // kv, (g + 1) * heads // kv):
                x = scale * (k @ q[r, h])
                m = x.max()
                p = np.exp(x - m)
                lse[r, h] = m + math.log(p.sum())
                p /= p.sum()
                out[r, h], spread[r, h] = p @ v, p @ np.abs(v)
                size[r, h] = abs(scale) * (np.abs(k) @ np.abs(q[r, h])).max()
                weights[r][g] += p
    return out, lse, spread, size, weights


def tree_places(table, n_pages, ps, lens, seen, n_draft=None, seq=None, max_len=None):
    """What the rows of trees see, for `attend`."""
    n, t, _ = seen.shape

    def places(r, g):
        b, i = divmod(r, t)
        s = b if seq is None else int(seq[b])
        length = max(0, min(int(lens[b]), table.shape[1] * ps if max_len is None else max_len, table.shape[1] * ps))
        d = t if n_draft is None else max(0, min(t, int(n_draft[b])))
        if i >= d or not 0 <= s < len(table):
            return []
        pos = list(range(length)) + [length + j for j in range(d) if seen[b, i, j]]
        at = [page_of(table, n_pages, ps, s, p) for p in pos]
        return [a for a in at if a is not None]
    return places


def row_places(table, n_pages, ps, lens, columns=None, seq=None, max_len=None):
    """What single rows see: all their tokens, or those of the listed columns."""
    def places(r, g):
        s = r if seq is None else int(seq[r])
        if not 0 <= s < len(table):
            return []
        n = max(0, min(int(lens[r]), table.shape[1] * ps if max_len is None else max_len, table.shape[1] * ps))
        if columns is None:
            pos = range(n)
        else:
            c = [int(x) for x in columns[r, g, :-(-n // ps)] if 0 <= x < table.shape[1]]
            pos = [x * ps + o for x in c for o in range(ps) if x * ps + o < n]
        at = [page_of(table, n_pages, ps, s, p) for p in pos]
        return [a for a in at if a is not None]
    return places


def keep(k_pool, v_pool, table, index, count, first=None, to=None):
    """Copies of the pools, changed; index(layer, s, head) is a list."""
    k, v = k_pool.copy(), v_pool.copy()
    layers, n_pages, kv, ps, _ = k.shape
    other = table if to is None else to
    for layer in range(layers):
        for s in range(len(table)):
            f = 0 if first is None else int(first[s])
            if f < 0:
                continue
            for g in range(kv):
                for j, i in enumerate(index(layer, s, g)[:max(0, int(count[s]))]):
                    if i < 0 or (to is None and i <= j):
                        continue
                    a, b = page_of(table, n_pages, ps, s, f + int(i)), page_of(other, n_pages, ps, s, f + j)
                    if a is not None and b is not None:
                        k[layer, b[0], g, b[1]] = k_pool[layer, a[0], g, a[1]]
                        v[layer, b[0], g, b[1]] = v_pool[layer, a[0], g, a[1]]
    return k, v


def trim(table, ref, lens, ps):
    table, ref = table.copy(), ref.copy()
    for s, n in enumerate(lens):
        for c in range(-(-max(0, int(n)) // ps), table.shape[1]):
            if 0 <= table[s, c] < len(ref):
                ref[table[s, c]] -= 1
            table[s, c] = -1
    return table, ref


def page_bounds(k_pages, table, lens, n_new, bounds):
    out = bounds.copy()
    n_pages, kv, ps, _ = k_pages.shape
    for s, n in enumerate(lens):
        n = max(0, min(int(n), table.shape[1] * ps))
        for c in range(max(0, n - n_new) // ps, -(-n // ps)):
            p = int(table[s, c])
            if not 0 <= p < n_pages or n_new == 0:
                continue
            keys = k_pages[p, :, :min(ps, n - c * ps)]
            none = np.isnan(keys).all(1)
            out[p, :, 0] = np.where(none, np.nan, np.where(np.isnan(keys), np.inf, keys).min(1))
            out[p, :, 1] = np.where(none, np.nan, np.where(np.isnan(keys), -np.inf, keys).max(1))
    return out


def page_scores(q, bounds):
    """q [heads of a kv head, hd], bounds [n, 2, hd]: [n]."""
    total = np.zeros(len(bounds))
    for x in q:
        with np.errstate(invalid="ignore"):
            a = np.maximum(x * bounds[:, 0], x * bounds[:, 1])
        total += np.where(x == 0, 0.0, a).sum(1)
    return np.where(np.isnan(total), np.inf, total)


def select_pages(q, bounds, table, lens, ps, n_select, sinks=1, recent=1, seq=None, max_len=None):
    rows, heads, _ = q.shape
    n_pages, kv = bounds.shape[:2]
    out = np.full((rows, kv, n_select), -1, np.int32)
    for r in range(rows):
        s = r if seq is None else int(seq[r])
        if not 0 <= s < len(table):
            continue
        n = max(0, min(int(lens[r]), table.shape[1] * ps if max_len is None else max_len, table.shape[1] * ps))
        columns = -(-n // ps)
        there = [c for c in range(columns) if 0 <= table[s, c] < n_pages]
        for g in range(kv):
            score = page_scores(q[r, g * heads // kv:(g + 1) * heads // kv], bounds[table[s, there], g])
            rank = {c: (0, -x, c) for c, x in zip(there, score)}
            for c in there:
                if c < sinks or c >= columns - recent:
                    rank[c] = (-1, 0, c)
            chosen = sorted(sorted(there, key=lambda c: rank[c])[:n_select])
            out[r, g, :len(chosen)] = chosen
    return out


def evict(weight, lens, budget, sinks=0, recent=1):
    n, kv, cap = weight.shape
    index, count = np.full((n, kv, budget), -1, np.int32), np.zeros(n, np.int32)
    out = np.zeros(weight.shape)
    for s in range(n):
        m = max(0, min(int(lens[s]), cap))
        count[s] = min(m, budget)
        for g in range(kv):
            def rank(j):
                w = weight[s, g, j]
                fixed = j < sinks or j >= m - recent
                return (-1, 0, j) if fixed else (0, -np.inf if np.isnan(w) else -w, j)
            kept = sorted(sorted(range(m), key=rank)[:budget])
            index[s, g, :len(kept)] = kept
            out[s, g, :len(kept)] = weight[s, g, kept]
    return index, count, out
