"""Inputs and error bounds shared by the tests of trees, chosen pages and
eviction."""
import numpy as np

from tests.paged_common import HALF_STEP


def random_tree(rng, draft, roots=1, wide=4):
    """Parents of a tree in which every node comes after its parent."""
    parent = np.full(draft, -1)
    for i in range(roots, draft):
        parent[i] = rng.integers(max(0, i - 2 * wide), i)
    return parent


def span_bounds(keys, spread, size, out, lse, hd, dtype):
    """Elementwise bounds of (out, lse) against float64, for rows of at most
    `keys` keys.

    A score is a sum of hd products, each and each partial sum off by 2^-24 of
    at most `size` (the largest sum |q k| scale), scaled and taken to powers of
    two: |ds| <= (hd + 4) 2^-24 size.  A weight is off by that on both sides of
    its quotient and by 2^-22 in its power; it reaches the products with all its
    bits.  A tile's keys are added one after the other in the worst case, and
    the tiles of a split after them, then 4 waves and at most 64 splits: fewer
    than keys + 128 additions, each off by 2^-24 of the spread (sum of p |v|).
    The output is rounded once."""
    ds = (hd + 4) * 2.0 ** -24 * size
    sums = (keys + 128) * 2.0 ** -24
    p = 2 * ds + 2.0 ** -21 + 2 * sums
    tol = p[..., None] * spread + (HALF_STEP[dtype] * 1.01) * np.abs(out) + 1e-30
    finite = np.where(np.isfinite(lse), np.abs(lse), 0.0)
    return tol, ds + 2.0 ** -21 + sums + 2.0 ** -22 * (finite + size)


def check(got, want, keys, hd, dtype):
    """(out, lse) as float64 arrays against `trees.attend`'s answer."""
    out, lse, spread, size = want[:4]
    tol, ltol = span_bounds(keys, spread, size, out, lse, hd, dtype)
    g, l = got
    assert np.array_equal(np.isneginf(l), np.isneginf(lse))
    off = np.abs(g - out) / tol
    assert (off <= 1).all(), off.max()
    ok = np.isfinite(lse)
    off = np.abs(l[ok] - lse[ok]) / ltol[ok]
    assert (off <= 1).all(), off.max()
