"""GPU: bounds of pages, the pages that a row reads, and attention over them,
against float64."""
import numpy as np
import pytest

from oracle import trees as ref
from tests.gpu_common import torch_cuda
from tests.paged_common import dtype_of, host, ints, normal, random_table
from tests.trees_common import check

pytestmark = pytest.mark.gpu


def same_bounds(got, want):
    got = host(got)
    assert np.array_equal(got, want, equal_nan=True), np.argwhere(got != want)[:5]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,page,kv", [(32, 1, 3), (64, 16, 2), (128, 8, 1), (128, 256, 2), (64, 1024, 1)])
def test_bounds(dtype, hd, page, kv):
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(hd + page)
    lens = np.array([1, 0, page, page + 1, 3 * page - 1, 700])
    table, n = random_table(rng, lens, page)
    table[5, 0] = -1
    k, k64 = normal(rng, (n, kv, page, hd), dtype)
    zero = np.zeros((n, kv, 2, hd))
    same_bounds(paged.page_bounds(k, ints(table), ints(lens)), ref.page_bounds(k64, table, lens, 1 << 30, zero))
    for n_new in (0, 1, 2, page, page + 1, 699, 5000):
        old, old64 = normal(rng, (n, kv, 2, hd), dtype)
        assert paged.page_bounds(k, ints(table), ints(lens), n_new=n_new, out=old) is old
        same_bounds(old, ref.page_bounds(k64, table, lens, n_new, old64))


def test_bounds_of_keys_that_are_not_finite():
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(5)
    table, n = random_table(rng, [20, 37], 8)
    for dtype in ("bf16", "f32"):
        k = rng.standard_normal((n, 2, 8, 32))
        k[rng.random(k.shape) < 0.3] = np.nan
        k[rng.random(k.shape) < 0.05] = np.inf
        k[rng.random(k.shape) < 0.05] = -np.inf
        k[table[0, 0], :, :, 3] = np.nan
        t = torch.from_numpy(k).to(dtype_of(dtype)).cuda()
        # lengths past the table and below 0
        for lens in ([20, 37], [2 ** 31 - 1, -5]):
            same_bounds(paged.page_bounds(t, ints(table), ints(lens)),
                        ref.page_bounds(host(t), table, lens, 1 << 30, np.zeros((n, 2, 2, 32))))


class Case:
    def __init__(self, seed, dtype, hd, H, kv, page, lens):
        rng = np.random.default_rng(seed)
        self.rng, self.dtype, self.hd, self.page, self.lens = rng, dtype, hd, page, np.array(lens)
        self.table, n = random_table(rng, lens, page)
        self.k, self.k64 = normal(rng, (n, kv, page, hd), dtype)
        self.v, self.v64 = normal(rng, (n, kv, page, hd), dtype)
        self.q, self.q64 = normal(rng, (len(lens), H, hd), dtype, 1.5)
        low, high = normal(rng, (n, kv, 1, hd), dtype), normal(rng, (n, kv, 1, hd), dtype)
        self.b64 = np.sort(np.concatenate((low[1], high[1]), 2), 2)
        self.bounds = torch_cuda().from_numpy(self.b64).to(dtype_of(dtype)).cuda()

    def select(self, n, **kw):
        from paper_2606_29223_amd import paged
        seq = kw.pop("seq", None)
        return paged.select_pages(kw.pop("q", self.q), self.bounds, ints(kw.pop("table", self.table)),
                                  ints(kw.pop("lens", self.lens)), self.page, n, seq=None if seq is None else ints(seq), **kw)

    def want(self, n, **kw):
        return ref.select_pages(self.q64, self.b64, kw.pop("table", self.table), kw.pop("lens", self.lens), self.page, n, **kw)

    def attend(self, columns, **kw):
        from paper_2606_29223_amd import paged
        seq = kw.pop("seq", None)
        return paged.sparse_attention(kw.pop("q", self.q), self.k, self.v, ints(kw.pop("table", self.table)),
                                      ints(kw.pop("lens", self.lens)), columns, seq=None if seq is None else ints(seq),
                                      return_lse=True, **kw)

    def check(self, got, columns, **kw):
        places = ref.row_places(kw.pop("table", self.table), len(self.k64), self.page, kw.pop("lens", self.lens), host(columns),
                                kw.pop("seq", None))
        check([host(t) for t in got], ref.attend(self.q64, self.k64, self.v64, places, **kw),
              columns.shape[2] * self.page, self.hd, self.dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,H,kv,page", [(32, 4, 4, 1), (64, 6, 2, 8), (128, 16, 1, 16), (128, 10, 5, 4), (64, 64, 1, 32)])
@pytest.mark.parametrize("n,sinks,recent", [(1, 0, 0), (1, 0, 1), (2, 1, 1), (7, 0, 0), (20, 3, 4), (300, 1, 1)])
def test_selection_and_attention(dtype, hd, H, kv, page, n, sinks, recent):
    torch_cuda()
    c = Case(hd + page + n, dtype, hd, H, kv, page, [1, 0, page, 5 * page - 1, 20 * page + 1, 257 * page])
    got = c.select(n, sinks=sinks, recent=recent)
    assert np.array_equal(host(got), c.want(n, sinks=sinks, recent=recent))
    assert np.array_equal(host(c.select(n, sinks=sinks, recent=recent, max_len=257 * page)), host(got))
    c.check(c.attend(got), got)


def test_ties_go_to_the_first():
    """Pages of equal bounds, and bounds of zeros: the lowest columns."""
    torch_cuda()
    c = Case(1, "bf16", 64, 8, 2, 16, [1600, 1590, 320])
    for group in (1, 7, 1000):
        same = c.table[0] // 1
        for s in range(3):
            for i, p in enumerate(c.table[s]):
                if p >= 0:
                    c.b64[p] = c.b64[c.table[s, i // group % 3]]
        c.bounds.copy_(torch_cuda().from_numpy(c.b64))
        assert len(same)
        for n in (1, 5, 33, 99):
            assert np.array_equal(host(c.select(n, sinks=0, recent=0)), c.want(n, sinks=0, recent=0))
    c.b64[:] = 0
    c.bounds.zero_()
    assert np.array_equal(host(c.select(40)), c.want(40))


def test_scores_that_are_not_finite():
    """Infinite bounds, NaN and zeros in the queries."""
    torch = torch_cuda()
    c = Case(2, "f32", 32, 4, 2, 4, [400, 399])
    p = c.table[0]
    c.b64[p[5], 0, 1] = np.inf
    c.b64[p[6], 0, 0, 3] = -np.inf
    c.b64[p[7], 1] = -np.inf
    c.b64[p[9], 1, 0], c.b64[p[9], 1, 1] = np.inf, -np.inf      # a page of NaN keys
    c.q64[0, :, 3] = 0
    c.q64[0, 0, 4] = -0.0
    c.q64[1, 1, 0] = np.nan
    c.bounds.copy_(torch.from_numpy(c.b64))
    c.q.copy_(torch.from_numpy(c.q64))
    for n in (3, 10, 50):
        assert np.array_equal(host(c.select(n)), c.want(n))


def test_missing_pages_lengths_and_sequences():
    torch_cuda()
    c = Case(3, "bf16", 64, 8, 2, 8, [500, 400, 300, 200, 100])
    t, n = c.table.copy(), len(c.k64)
    t[0, 0] = -1
    t[1, ::2] = n
    t[2, 37] = 2 ** 31 - 1
    t[3, :] = -2 ** 31
    got = c.select(12, table=t, sinks=2, recent=3)
    assert np.array_equal(host(got), c.want(12, table=t, sinks=2, recent=3))
    c.check(c.attend(got, table=t), got, table=t)
    seq, lens = np.array([4, 7, -1, 0, 2]), np.array([2 ** 31 - 1, 5, 6, -9, 33])
    got = c.select(12, seq=seq, lens=lens)
    assert np.array_equal(host(got), c.want(12, seq=seq, lens=lens))
    c.check(c.attend(got, seq=seq, lens=lens), got, seq=seq, lens=lens)
    assert (host(c.select(12, max_len=0)) == -1).all()
    assert np.array_equal(host(c.select(12, max_len=99)), c.want(12, max_len=99))


def test_long_tables():
    """Thousands of columns, nearly equal scores among them."""
    torch_cuda()
    c = Case(4, "bf16", 32, 4, 2, 1, [9000, 4097, 70])
    c.b64 = np.round(c.b64 * 2) / 2
    c.bounds.copy_(torch_cuda().from_numpy(c.b64))
    for n in (2, 64, 2000, 9000):
        got = c.select(n)
        assert np.array_equal(host(got), c.want(n))
    c.check(c.attend(got), got)


def test_columns_of_the_callers_own():
    """Any order, twice the same, outside the table, more than the row has."""
    torch_cuda()
    c = Case(6, "bf16", 64, 8, 2, 16, [300, 40, 161])
    columns = np.full((3, 2, 25), -1)
    columns[0] = c.rng.integers(0, 19, (2, 25))
    columns[0, 0, 3], columns[0, 1, 0] = 2 ** 31 - 1, -2 ** 31
    columns[1] = 2
    columns[2, 0, ::2] = 10
    got = ints(columns)
    c.check(c.attend(got), got)
    for scale in (0.5, -0.1):
        c.check(c.attend(got, scale=scale), got, scale=scale)


def test_strided_queries_and_outputs():
    torch = torch_cuda()
    c = Case(7, "bf16", 64, 6, 2, 16, [300, 40])
    columns = c.select(4)
    want = [host(t) for t in c.attend(columns)]
    x = torch.full((2, 9, 71), 9.0, dtype=torch.bfloat16, device="cuda")
    q = x[:, 2:8, 3:67]
    q.copy_(c.q)
    assert np.array_equal(host(c.select(4, q=q)), host(columns))
    y = torch.full((2, 9, 71), 9.0, dtype=torch.bfloat16, device="cuda")
    got = c.attend(columns, q=q, out=y[:, 2:8, 3:67])
    assert all(np.array_equal(a, host(b)) for a, b in zip(want, got))
    y[:, 2:8, 3:67] = 9.0
    assert (y == 9.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,page", [(64, 1), (128, 2), (32, 4)])
def test_lists_of_more_columns_than_a_wave_holds(dtype, hd, page):
    """Lists on both sides of 64 columns, in any order, some of them twice or none
    of the table's, some of their pages missing."""
    torch_cuda()
    n = 300
    c = Case(hd, dtype, hd, 8, 2, page, [61 * page, 64 * page, 65 * page + 1, 300 * page, 40 * page - 1, 0])
    columns = c.rng.integers(-2, 310, (6, 2, n))
    t = c.table.copy()
    t[3, 5::7] = -1
    columns = ints(columns)
    c.check(c.attend(columns, table=t), columns, table=t)
