"""The operators over a paged key/value cache (include/dex.h), from their
definitions in float64 and one thing at a time: the library's kernels are
tested against these.  Arrays are numpy; cache rows are
[n_pages, n_kv_heads, page_size, head_dim]."""
from __future__ import annotations

import math

import numpy as np


def frequencies(rot_dim, theta=1e4, scaling=None, factor=1.0, original=0.0, slow=1.0, fast=32.0):
    """Radians a position of each pair."""
    out = []
    for i in range(rot_dim // 2):
        base = theta * factor ** (rot_dim / (rot_dim - 2)) if scaling == "base" else theta
        f = base ** (-2 * i / rot_dim)
        if scaling == "linear":
            f /= factor
        if scaling == "bands":
            n = original * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (n - slow) / (fast - slow)))
            f = keep * f + (1 - keep) * f / factor
        out.append(f)
    return np.array(out)


def rotate(x, pos, freq, interleaved=False, amplitude=1.0, inverse=False):
    """x [rows, heads, head_dim] turned to positions pos [rows]."""
    x = np.asarray(x, dtype=np.float64)
    y = x.copy()
    n = len(freq)
    for r, p in enumerate(pos):
        for i, f in enumerate(freq):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
            t = -float(p) * f if inverse else float(p) * f
            c, s = amplitude * math.cos(t), amplitude * math.sin(t)
            y[r, :, a] = x[r, :, a] * c - x[r, :, b] * s
            y[r, :, b] = x[r, :, b] * c + x[r, :, a] * s
    return y


def page_of(table, n_pages, page_size, seq, pos):
    """(page, slot) of a position, or None."""
    if not 0 <= seq < len(table) or pos < 0 or pos // page_size >= table.shape[1]:
        return None
    page = int(table[seq, pos // page_size])
    return (page, pos % page_size) if 0 <= page < n_pages else None


def attention(q, k_pages, v_pages, table, lens, seq=None, max_len=None, scale=None, window=0):
    """(out, lse, spread): spread[r, h, d] = sum_j p_j |v_jd|, and the largest
    sum |q_i k_i| * scale over the keys (for error bounds) as a fourth."""
    rows, heads, hd = q.shape
    n_pages, kv, ps, _ = k_pages.shape
    q, k_pages, v_pages = (np.asarray(t, dtype=np.float64) for t in (q, k_pages, v_pages))
    scale = hd ** -0.5 if scale is None else scale
    out, lse, spread = np.zeros(q.shape), np.full((rows, heads), -np.inf), np.zeros(q.shape)
    size = np.zeros((rows, heads))
    for r in range(rows):
        s = r if seq is None else int(seq[r])
        n = int(lens[r]) if max_len is None else min(int(lens[r]), max_len)
        n = min(n, table.shape[1] * ps)
        lo = max(0, n - window) if window else 0
        at = [page_of(table, n_pages, ps, s, j) for j in range(lo, n)]
        at = [a for a in at if a is not None]
        if not at:
            continue
        page, slot = np.array(at).T
        for h in range(heads):
            g = h // (heads // kv)
            k, v = k_pages[page, g, slot], v_pages[page, g, slot]
            x = scale * (k @ q[r, h])
            m = x.max()
            p = np.exp(x - m)
            lse[r, h] = m + math.log(p.sum())
            p /= p.sum()
            out[r, h], spread[r, h] = p @ v, p @ np.abs(v)
            size[r, h] = scale * (np.abs(k) @ np.abs(q[r, h])).max()
    return out, lse, spread, size


def fork(table, ref, lens, parent):
    table, ref, lens = table.copy(), ref.copy(), lens.copy()
    old, old_len = table.copy(), lens.copy()
    for row in old:
        for p in row:
            if 0 <= p < len(ref):
                ref[p] -= 1
    for s, f in enumerate(parent):
        if 0 <= f < len(old):
            table[s], lens[s] = old[f], old_len[f]
            for p in old[f]:
                if 0 <= p < len(ref):
                    ref[p] += 1
        else:
            table[s], lens[s] = -1, 0
    return table, ref, lens


def reserve(table, ref, lens, n_new, page_size):
    """One sequence after another; all or none."""
    t, r, n = table.copy(), ref.copy(), lens.copy()
    S = len(table)
    free = [p for p in range(len(ref)) if ref[p] == 0]
    taken, wanted, bad = 0, 0, 0
    pos, src, dst, tok = np.full(S, -1), [], [], []
    for s in range(S):
        add = max(0, int(n_new[s]))
        if add == 0:
            continue
        if lens[s] < 0 or lens[s] + add > t.shape[1] * page_size:
            bad = 1
            continue
        cols = list(range(-(-int(lens[s]) // page_size), -(-int(lens[s] + add) // page_size)))
        part = int(lens[s]) % page_size
        old = -1
        if part:
            c = int(lens[s]) // page_size
            old = int(t[s, c]) if 0 <= t[s, c] < len(ref) else -1
            if old < 0 or r[old] > 1:
                cols.insert(0, c)
            else:
                old = -1
        for c in cols:
            wanted += 1
            if taken < len(free):
                t[s, c] = free[taken]
                r[free[taken]] = 1
                taken += 1
            else:
                t[s, c] = -1                      # refused below
        if part and old >= 0:
            r[old] -= 1
            src.append(old)
            dst.append(int(t[s, cols[0]]))
            tok.append(part)
        pos[s] = lens[s]
        n[s] += add
    short = max(0, wanted - len(free))
    if short or bad:
        none = np.full(S, -1)
        return table, ref, lens, none, none, none, np.zeros(S, int), [0, 0, short, bad]
    fill = S - len(src)
    return (t, r, n, pos, np.array(src + [-1] * fill), np.array(dst + [-1] * fill), np.array(tok + [0] * fill),
            [len(src), wanted, 0, 0])


def compact(table, ref):
    n = len(ref)
    used = int((ref > 0).sum())
    movers = [p for p in range(used, n) if ref[p] > 0]
    holes = [p for p in range(used) if ref[p] <= 0]
    new = np.array([p if ref[p] > 0 else -1 for p in range(n)])
    r = ref.copy()
    for a, b in zip(movers, holes):
        new[a] = b
        r[b], r[a] = ref[a], 0
    t = np.array([[new[p] if 0 <= p < n else -1 for p in row] for row in table])
    fill = [-1] * (n // 2 - len(movers))
    return t, r, new, np.array(movers + fill, int), np.array(holes + fill, int), [len(movers), used, 0, 0]


def beam_select(logits, scores, n_out, done=None, eos=-1):
    requests, beams = scores.shape
    vocab = logits.shape[1]
    x = np.asarray(logits, dtype=np.float64)
    parent, token = np.zeros((requests, n_out), int), np.zeros((requests, n_out), int)
    score, ends = np.zeros((requests, n_out)), np.zeros((requests, n_out), bool)
    for r in range(requests):
        total = np.full((beams, vocab), -np.inf)
        for b in range(beams):
            s, row = float(scores[r, b]), x[r * beams + b]
            if not math.isfinite(s):
                continue
            if done is not None and done[r, b]:
                total[b, eos] = s
                continue
            m = row.max() if not np.isnan(row).any() else np.nan
            if math.isfinite(m):
                with np.errstate(divide="ignore"):
                    total[b] = s + (row - (m + math.log(np.exp(row - m).sum())))
        order = sorted(range(beams * vocab), key=lambda i: (-total.flat[i], i))[:n_out]
        for k, i in enumerate(order):
            b, t = divmod(i, vocab)
            parent[r, k], token[r, k], score[r, k] = r * beams + b, t, total[b, t]
            ends[r, k] = (done is not None and done[r, b]) or t == eos
    return parent, token, score, ends
