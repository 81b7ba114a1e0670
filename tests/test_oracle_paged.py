"""The float64 references of the paged-cache operators against closed forms and
invariants, so that the GPU tests compare with something that is right."""
import math

import numpy as np
import pytest

from oracle import paged as ref


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_complex_product_and_turns_back(interleaved):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 3, 16))
    pos = np.array([0, 1, -7, 1000, 123456])
    f = ref.frequencies(8)
    y = ref.rotate(x, pos, f, interleaved)
    a, b = (slice(0, 8, 2), slice(1, 8, 2)) if interleaved else (slice(0, 4), slice(4, 8))
    z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * pos[:, None, None] * f)
    np.testing.assert_allclose(y[..., a] + 1j * y[..., b], z, atol=1e-12)
    np.testing.assert_array_equal(y[..., 8:], x[..., 8:])
    np.testing.assert_allclose(ref.rotate(y, pos, f, interleaved, inverse=True), x, atol=1e-12)


def test_the_inverse_is_the_gradient():
    """<g, R x> has the gradient R' g: by differences in every coordinate."""
    rng = np.random.default_rng(2)
    x, g = rng.standard_normal((2, 1, 8)), rng.standard_normal((2, 1, 8))
    pos, f = np.array([3, 77]), ref.frequencies(6)
    want = ref.rotate(g, pos, f, amplitude=1.25, inverse=True)
    for i in range(x.size):
        d = np.zeros(x.size)
        d[i] = 0.5
        up, down = (float((g * ref.rotate(x + t * d.reshape(x.shape), pos, f, amplitude=1.25)).sum()) for t in (1, -1))
        assert abs(up - down - want.flat[i]) < 1e-12


def test_scaled_frequencies():
    plain = ref.frequencies(64)
    assert plain[0] == 1.0 and abs(plain[16] - 1e-2) < 1e-15
    np.testing.assert_allclose(ref.frequencies(64, scaling="linear", factor=4), plain / 4)
    base = ref.frequencies(64, scaling="base", factor=8)
    assert base[0] == 1.0 and abs(base[-1] - plain[-1] / 8) < 1e-15 * plain[-1]   # the lowest is divided by it
    bands = ref.frequencies(64, scaling="bands", factor=16, original=8192, slow=1, fast=32)
    turns = 8192 * plain / (2 * math.pi)
    np.testing.assert_allclose(bands[turns >= 32], plain[turns >= 32])
    np.testing.assert_allclose(bands[turns <= 1], plain[turns <= 1] / 16)
    assert np.all(np.diff(bands) < 0)


def _holders(table, n):
    return np.bincount(table[table >= 0], minlength=n)


def test_pages_keep_their_counts_through_a_random_life():
    """Forks, growth and compaction over many steps: the counts stay the number
    of table rows that list a page, a written page has one holder, every
    position keeps the token written there, and nothing is lost."""
    rng = np.random.default_rng(3)
    S, C, P, ps = 6, 8, 40, 4
    table, counts, lens = np.full((S, C), -1), np.zeros(P, int), np.zeros(S, int)
    store = np.full((P, ps), -1)
    want = [[] for _ in range(S)]
    shorts = 0
    for step in range(300):
        parent = np.array([rng.choice([s, s, rng.integers(S), -1]) for s in range(S)])
        table, counts, lens = ref.fork(table, counts, lens, parent)
        want = [list(want[f]) if f >= 0 else [] for f in parent]
        add = np.where(lens < 24, rng.integers(0, 6, S), 0)
        before = table.copy()
        table, counts, lens, pos, src, dst, tok, state = ref.reserve(table, counts, lens, add, ps)
        shorts += state[2] > 0
        if state[2]:
            assert np.array_equal(table, before) and (pos == -1).all()
        for a, b, n in zip(src, dst, tok):
            if a >= 0:
                store[b, :n] = store[a, :n]
        for s in range(S):
            if pos[s] >= 0:
                for i in range(add[s]):
                    p, slot = ref.page_of(table, P, ps, s, pos[s] + i)
                    assert counts[p] == 1
                    store[p, slot] = step * 100 + s * 10 + i
                    want[s].append(step * 100 + s * 10 + i)
        if step % 7 == 0:
            table, counts, new, a, b, state = ref.compact(table, counts)
            for x, y in zip(a, b):
                if x >= 0:
                    store[y] = store[x]
            assert (counts[:state[1]] > 0).all() and (counts[state[1]:] == 0).all()
        assert np.array_equal(counts, _holders(table, P))
        for s in range(S):
            assert lens[s] == len(want[s])
            got = [store[ref.page_of(table, P, ps, s, j)] for j in range(lens[s])]
            assert got == want[s]
    assert shorts == 0


def test_last_writer_keeps_an_unheld_page():
    table, counts, lens = np.array([[0], [0], [0]]), np.array([3, 0, 0, 0]), np.array([2, 2, 2])
    t, r, n, pos, src, dst, tok, state = ref.reserve(table, counts, lens, np.ones(3, int), 4)
    assert t[:, 0].tolist() == [1, 2, 0] and r.tolist() == [1, 1, 1, 0] and state == [2, 2, 0, 0]
    assert src.tolist() == [0, 0, -1] and dst.tolist() == [1, 2, -1] and tok.tolist() == [2, 2, 0]
    # a fourth holder outside the table: everyone copies
    t, r, *_ = ref.reserve(table, np.array([4, 0, 0, 0]), lens, np.ones(3, int), 4)
    assert t[:, 0].tolist() == [1, 2, 3] and r.tolist() == [1, 1, 1, 1]
    # too few pages: nothing at all
    t, r, n, pos, *_, state = ref.reserve(table, np.array([4, 0, 1, 0]), lens, np.ones(3, int), 4)
    assert np.array_equal(t, table) and state == [0, 0, 1, 0] and (pos == -1).all()


def test_attention_special_cases():
    rng = np.random.default_rng(4)
    k, v = rng.standard_normal((2, 5, 2, 4, 8))
    q = rng.standard_normal((3, 4, 8))
    table = np.array([[3, 1], [-1, 2], [-1, -1]])
    out, lse, spread, _ = ref.attention(q, k, v, table, [1, 7, 5])
    np.testing.assert_allclose(out[0, 3], v[3, 1, 0])                  # one key
    np.testing.assert_allclose(lse[0, 3], q[0, 3] @ k[3, 1, 0] / math.sqrt(8))
    x = np.exp(k[2, 0, :3] @ q[1, 0] / math.sqrt(8))                   # a page is missing
    np.testing.assert_allclose(out[1, 0], x @ v[2, 0, :3] / x.sum())
    assert (out[2] == 0).all() and (lse[2] == -np.inf).all()           # no page at all
    window, *_ = ref.attention(q, k, v, table, [8, 0, 0], window=1)
    np.testing.assert_allclose(window[0, 0], v[1, 0, 3])


def test_beams_against_a_full_sort():
    rng = np.random.default_rng(5)
    x, s = rng.standard_normal((6, 11)), rng.standard_normal((2, 3))
    parent, token, score, _ = ref.beam_select(x, s, 3)
    logp = x - np.log(np.exp(x).sum(1, keepdims=True))
    total = (s.reshape(-1, 1) + logp).reshape(2, -1)
    order = np.argsort(-total, axis=1, kind="stable")[:, :3]
    assert np.array_equal(parent - np.array([[0], [3]]), order // 11) and np.array_equal(token, order % 11)
    np.testing.assert_allclose(score, np.take_along_axis(total, order, 1))
    done = np.array([[True, False, False], [False, False, True]])
    s2 = np.array([[5.0, -40, -40], [-np.inf, 0, -np.inf]])
    parent, token, score, ends = ref.beam_select(x, s2, 3, done=done, eos=4)
    assert (parent[0, 0], token[0, 0], score[0, 0], ends[0, 0]) == (0, 4, 5.0, True)
    assert (parent[1] == 4).all()                                      # the one live beam
