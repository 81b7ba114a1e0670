"""The float64 definitions of trees, page selection and eviction, pinned to
values worked out by hand and to brute force."""
import itertools

import numpy as np

from oracle import paged, trees


def test_a_tree_by_hand():
    #      0        5 (a second root)
    #    1   2
    #    3   4
    parent = np.array([[-1, 0, 0, 1, 2, -1]])
    seen, depth = trees.tree_mask(parent)
    assert depth.tolist() == [[0, 1, 1, 2, 2, 0]]
    assert seen[0].astype(int).tolist() == [[1, 0, 0, 0, 0, 0], [1, 1, 0, 0, 0, 0], [1, 0, 1, 0, 0, 0], [1, 1, 0, 1, 0, 0],
                                            [1, 0, 1, 0, 1, 0], [0, 0, 0, 0, 0, 1]]
    assert trees.words(seen)[0, :, 0].tolist() == [1, 3, 5, 11, 21, 32]
    token, target = np.array([[9, 4, 5, 6, 7, 9]]), np.array([[5, 6, 7, 1, 2, 3]])
    path, count, after = trees.tree_accept(parent, token, target)
    assert path.tolist() == [[0, 2, 4, -1, -1, -1]] and count[0] == 3 and after[0] == 2
    path, count, after = trees.tree_accept(parent, token, target, n_draft=[4])
    assert path.tolist() == [[0, 2, -1, -1, -1, -1]] and after[0] == 7
    path, count, after = trees.tree_accept(parent, token, target, root=[8])
    assert count[0] == 0 and after[0] == 8


def test_parents_that_are_none_are_roots():
    seen, depth = trees.tree_mask(np.array([[0, 1, 5, -7, 3]]))
    assert depth.tolist() == [[0, 0, 0, 0, 1]]


def test_words_past_64():
    seen = np.zeros((1, 130, 130), bool)
    seen[0, 5, [0, 63, 64, 129]] = True
    w = trees.words(seen).view(np.uint64)[0, 5]
    assert w.tolist() == [1 | 1 << 63, 1, 2]


def test_a_tree_without_drafts_is_the_rows_attention():
    rng = np.random.default_rng(0)
    k, v = rng.standard_normal((9, 2, 4, 8)), rng.standard_normal((9, 2, 4, 8))
    q, table, lens = rng.standard_normal((2, 4, 8)), np.array([[3, 1, -1], [0, 8, 2]]), [7, 11]
    a = paged.attention(q, k, v, table, lens)
    b = trees.attend(q, k, v, trees.row_places(table, 9, 4, lens))
    every = np.tile(np.arange(3), (2, 2, 1))
    c = trees.attend(q, k, v, trees.row_places(table, 9, 4, lens, columns=every))
    for x, y, z in zip(a, b, c):
        np.testing.assert_allclose(x, y, rtol=1e-13)
        np.testing.assert_allclose(x, z, rtol=1e-13)
    # weights of a kv head's two query heads add up to two
    np.testing.assert_allclose([w.sum() for r in b[4] for w in r], 2.0)


def test_a_drafted_token_sees_its_ancestors():
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((4, 1, 4, 8)), rng.standard_normal((4, 1, 4, 8))
    table = np.array([[2, 0, 1]])
    seen, _ = trees.tree_mask(np.array([[-1, 0, 0]]))
    places = trees.tree_places(table, 4, 4, [6], seen)
    assert places(2, 0) == [(2, 0), (2, 1), (2, 2), (2, 3), (0, 0), (0, 1), (0, 2), (1, 0)]


def test_scores_bound_every_key():
    rng = np.random.default_rng(2)
    keys, q = rng.standard_normal((5, 8, 16)), rng.standard_normal((3, 16))
    bounds = np.stack((keys.min(1), keys.max(1)), 1)
    score = trees.page_scores(q, bounds)
    assert (score >= (keys @ q.T).sum(2).max(1)).all()
    # the sum over heads of the largest product over all corners of the box
    small, x = bounds[0, :, :4], q[:, :4]
    best = sum(max(sum(a * small[c, d] for d, (a, c) in enumerate(zip(y, corner)))
                   for corner in itertools.product((0, 1), repeat=4)) for y in x)
    np.testing.assert_allclose(trees.page_scores(x, small[None])[0], best)


def test_selection_and_eviction_by_hand():
    q = np.array([[[1.0, 0.0]]])
    bounds = np.zeros((6, 1, 2, 2))
    bounds[:, 0, 1, 0] = [5, 1, 7, 7, 3, 2]
    table = np.array([[0, 1, 2, 3, 4, 5]])
    assert trees.select_pages(q, bounds, table, [11], 2, 4, 1, 1).tolist() == [[[0, 2, 3, 5]]]
    assert trees.select_pages(q, bounds, table, [11], 2, 3, 1, 1).tolist() == [[[0, 2, 5]]]       # a tie: the first
    assert trees.select_pages(q, bounds, table, [3], 2, 4, 1, 1).tolist() == [[[0, 1, -1, -1]]]
    w = np.array([[[1.0, 9.0, 2.0, 9.0, 0.5, 0.1, 4.0]]])
    index, count, out = trees.evict(w, [6], 4, 1, 1)
    assert index.tolist() == [[[0, 1, 3, 5]]] and count.tolist() == [4]
    assert out[0, 0].tolist() == [1.0, 9.0, 9.0, 0.1, 0, 0, 0]


def test_keep_and_trim_by_hand():
    k = np.arange(24.0).reshape(1, 4, 1, 2, 3)
    table = np.array([[2, 0, 3, -1]])
    got, _ = trees.keep(k, k, table, lambda *_: [0, 2, 3], [3], first=[1])
    # positions 1, 3, 4 of the sequence move to 1, 2, 3
    assert got[0, 2, 0, 1].tolist() == k[0, 2, 0, 1].tolist()
    assert got[0, 0, 0, 0].tolist() == k[0, 0, 0, 1].tolist()
    assert got[0, 0, 0, 1].tolist() == k[0, 3, 0, 0].tolist()
    t, r = trees.trim(table, np.array([1, 0, 1, 2]), [4], 2)
    assert t.tolist() == [[2, 0, -1, -1]] and r.tolist() == [1, 0, 1, 1]
