"""GPU: page tables (fork and free, reserve, compact) and page copies against
the one-at-a-time reference, exactly."""
import numpy as np
import pytest

from oracle import paged as ref
from tests.gpu_common import torch_cuda
from tests.paged_common import host, ints, normal

pytestmark = pytest.mark.gpu


def _life(rng, S, C, P, ps, extra=0):
    """A reachable state: tables of random sequences that share some pages."""
    table, counts, lens = np.full((S, C), -1), np.zeros(P, int), np.zeros(S, int)
    counts[rng.permutation(P)[:extra]] += 1               # held by someone else
    for _ in range(4):
        want = np.minimum(rng.integers(0, C * ps // 4 + 1, S), C * ps - lens)
        out = ref.reserve(table, counts, lens, want, ps)
        if not out[7][2]:
            table, counts, lens = out[:3]
        parent = np.where(rng.random(S) < 0.4, rng.integers(0, S, S), np.arange(S))
        parent[rng.random(S) < 0.1] = -1
        table, counts, lens = ref.fork(table, counts, lens, parent)
    return table, counts, lens


SHAPES = [(1, 1, 1, 1), (1, 7, 9, 4), (8, 60, 300, 16), (3, 5, 17, 1), (64, 33, 2500, 8), (1024, 20, 30000, 2),
          (1000, 3, 9, 64), (37, 300, 20000, 1), (2, 4000, 70000, 4)]


@pytest.mark.parametrize("S,C,P,ps", SHAPES)
@pytest.mark.parametrize("in_place", [False, True])
def test_fork(S, C, P, ps, in_place):
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(S + C)
    table, counts, lens = _life(rng, S, C, P, ps)
    for parent in (np.arange(S), rng.integers(0, S, S), np.full(S, -1), np.zeros(S, int),
                   np.where(rng.random(S) < 0.5, np.arange(S), rng.choice([-1, S, -2 ** 31, 2 ** 31 - 1], S))):
        t, r, n = ints(table), ints(counts), ints(lens)
        got = paged.fork(t, r, n, ints(parent), out=(t, r, n) if in_place else None)
        for a, b in zip(got, ref.fork(table, counts, lens, parent)):
            assert np.array_equal(host(a), b)
        if not in_place:                                  # the inputs are as they were
            assert np.array_equal(host(t), table) and np.array_equal(host(r), counts) and np.array_equal(host(n), lens)


def _check_reserve(paged, table, counts, lens, n_new, ps):
    t, r, n = ints(table), ints(counts), ints(lens)
    got = paged.reserve(t, r, n, ints(n_new), ps)
    want = ref.reserve(table, counts, lens, n_new, ps)
    for name, a, b in zip(("table", "ref", "lens", "pos", "src", "dst", "tokens", "state"), (t, r, n, *got), want):
        assert np.array_equal(host(a), np.array(b)), (name, host(got.state), want[7])
    return want


@pytest.mark.parametrize("S,C,P,ps", SHAPES)
def test_reserve(S, C, P, ps):
    torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(S * 7 + C)
    table, counts, lens = _life(rng, S, C, P, ps, extra=P // 10)
    room = C * ps - lens
    for n_new in (np.ones(S, int), np.zeros(S, int), rng.integers(-2, 3, S), rng.integers(0, 2 * ps + 2, S), room,
                  room // 2, np.where(np.arange(S) == S - 1, room + 1, 0)):
        _check_reserve(paged, table, counts, lens, np.minimum(n_new, room + 1), ps)


def test_reserve_takes_more_pages_than_it_keeps_in_lds():
    torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(3)
    counts = (rng.random(40000) < 0.4).astype(int)
    table, lens = np.full((16, 1500), -1), np.zeros(16, int)
    free = int((counts == 0).sum())
    want = _check_reserve(paged, table, counts, lens, np.full(16, 1500), 1)          # 24000 pages or none
    assert (want[7][2] > 0) == (free < 24000)
    want = _check_reserve(paged, table, counts, lens, np.full(16, 1201), 1)
    assert want[7][:3] == [0, 16 * 1201, 0]
    exact = np.full(16, free // 16)
    exact[0] += free - exact.sum()
    if exact.max() <= 1500:
        assert _check_reserve(paged, table, counts, lens, exact, 1)[7][1] == free    # the last free page too
        exact[3] += 1
        assert _check_reserve(paged, table, counts, lens, exact, 1)[7][2] == 1       # and one too many


def test_reserve_shared_pages_and_bad_states():
    """Many writers of one page, with and without another holder; a partly
    filled page that is missing; lengths below 0 and past the table."""
    torch_cuda()
    from paper_2606_29223_amd import paged
    for holders in (9, 10, 1, 0):
        table = np.full((9, 4), -1)
        table[:, 0] = 5
        counts = np.zeros(64, int)
        counts[5] = holders
        for n_new in (np.ones(9, int), np.array([0, 1, 0, 1, 1, 0, 0, 9, 1])):
            _check_reserve(paged, table, counts, np.full(9, 3), n_new, 8)
    table = np.array([[-1, 2], [99, -1], [0, -1], [1, -1]])
    counts = np.array([1, 1, 1, 0, 0, 0])
    _check_reserve(paged, table, counts, np.array([3, 5, 8, 2]), np.ones(4, int), 8)
    _check_reserve(paged, table, counts, np.array([3, -5, 8, 2]), np.array([1, 0, 1, 1]), 8)
    _check_reserve(paged, table, counts, np.array([3, -5, 8, 2]), np.array([1, 1, 1, 1]), 8)
    _check_reserve(paged, table, counts, np.array([3, 17, 8, 2 ** 31 - 1]), np.array([1, 0, 1, 2 ** 31 - 1]), 8)


@pytest.mark.parametrize("S,C,P,ps", SHAPES)
@pytest.mark.parametrize("in_place", [False, True])
def test_compact(S, C, P, ps, in_place):
    torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(S * 3 + P)
    table, counts, lens = _life(rng, S, C, P, ps, extra=P // 5)
    t, r = ints(table), ints(counts)
    out = None if in_place else (ints(table * 0), ints(counts * 0))
    got = paged.compact(t, r, out=out)
    want = ref.compact(table, counts)
    for name, a, b in zip(("table", "ref", "new", "src", "dst", "state"), (*(out or (t, r)), *got), want):
        assert np.array_equal(host(a), np.array(b)), name


@pytest.mark.parametrize("dtype,hd,kv,page,layers", [("bf16", 128, 8, 16, 3), ("bf16", 8, 1, 1, 1), ("f32", 64, 12, 32, 2),
                                                     ("bf16", 64, 3, 1024, 2), ("f32", 4, 5, 2, 40)])
def test_copy(dtype, hd, kv, page, layers):
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(hd + page)
    P, n = 30, 9
    k, k64 = normal(rng, (layers, P, kv, page, hd), dtype)
    v, v64 = normal(rng, (layers, P, kv, page, hd), dtype)
    ids = rng.permutation(P)
    src, dst = ids[:n].copy(), ids[n:2 * n].copy()
    src[3] = dst[3]                                       # onto itself
    tokens = rng.integers(0, page + 1, n)
    tokens[:3] = (page, 0, page + 5)
    for count, tok in ((None, None), (4, tokens), (0, None), (100, tokens), (-1, tokens), (None, tokens)):
        a, b = k.clone(), v.clone()
        paged.copy(a, b, ints(src), ints(dst), None if count is None else ints([count]), None if tok is None else ints(tok))
        for got, was in ((host(a), k64), (host(b), v64)):
            want = was.copy()
            for i in range(n if count is None else max(0, min(n, count))):
                m = page if tok is None else max(0, min(page, tok[i]))
                want[:, dst[i], :, :m] = was[:, src[i], :, :m]
            assert np.array_equal(got, want), (count, tok)
    src[0], dst[1], src[2], dst[4] = -1, P, 2 ** 31 - 1, -2 ** 31
    a, b = k.clone(), v.clone()
    paged.copy(a, b, ints(src), ints(dst))
    want = k64.copy()
    for i in (3, 5, 6, 7, 8):
        want[:, dst[i]] = k64[:, src[i]]
    assert np.array_equal(host(a), want)
