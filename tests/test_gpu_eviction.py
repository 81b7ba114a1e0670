"""GPU: attention that adds up what each key was given, against float64, and the
keys that stay by those totals."""
import numpy as np
import pytest

from oracle import trees as ref
from tests.gpu_common import torch_cuda
from tests.paged_common import host, ints, normal, random_table
from tests.trees_common import check, span_bounds

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, seed, dtype, hd, H, kv, page, lens, extra=0):
        rng = np.random.default_rng(seed)
        self.rng, self.dtype, self.hd, self.page, self.lens = rng, dtype, hd, page, np.array(lens)
        self.table, n = random_table(rng, lens, page)
        self.k, self.k64 = normal(rng, (n, kv, page, hd), dtype)
        self.v, self.v64 = normal(rng, (n, kv, page, hd), dtype)
        self.q, self.q64 = normal(rng, (len(lens), H, hd), dtype, 1.5)
        self.cap = self.table.shape[1] * page + extra
        self.weight, self.w64 = normal(rng, (len(lens), kv, self.cap), "f32")
        self.weight.abs_()
        self.w64 = np.abs(self.w64)

    def run(self, **kw):
        from paper_2606_29223_amd import paged
        seq = kw.pop("seq", None)
        return paged.weigh(kw.pop("q", self.q), self.k, self.v, ints(kw.pop("table", self.table)),
                           ints(kw.pop("lens", self.lens)), kw.pop("weight", self.weight),
                           seq=None if seq is None else ints(seq), return_lse=True, **kw)

    def check(self, got, total, **kw):
        table, lens = kw.pop("table", self.table), kw.pop("lens", self.lens)
        seq, max_len = kw.pop("seq", None), kw.pop("max_len", None)
        want = ref.attend(self.q64, self.k64, self.v64,
                          ref.row_places(table, len(self.k64), self.page, lens, seq=seq, max_len=max_len), **kw)
        keys = self.cap
        check([host(t) for t in got], want, keys, self.hd, self.dtype)
        rows, kv, _ = self.w64.shape
        G = self.q64.shape[1] // kv
        for r in range(rows):
            s = r if seq is None else int(seq[r])
            n = max(0, min(int(lens[r]), table.shape[1] * self.page if max_len is None else max_len, table.shape[1] * self.page))
            if not 0 <= s < len(table):
                n = 0
            there = [j for j in range(n) if 0 <= table[s, j // self.page] < len(self.k64)]
            for g in range(kv):
                w = np.zeros(self.cap)
                w[there] = want[4][r][g]
                # a weight is off as in the outputs, by two scores, its power and the
                # sum below it; G of them are added, and to the total
                ds = (self.hd + 4) * 2.0 ** -24 * want[3][r, g * G:(g + 1) * G].max()
                rel = 2 * ds + 2.0 ** -21 + 2 * (keys + 128) * 2.0 ** -24 + G * 2.0 ** -24
                sums = self.w64[r, g] + w
                off = np.abs(host(total)[r, g] - sums) - (rel * w + 2.0 ** -24 * np.abs(sums))
                assert (off <= 0).all(), off.max()
                assert np.array_equal(host(total)[r, g, n:], self.w64[r, g, n:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("H,kv,page", [(4, 4, 1), (6, 2, 8), (16, 1, 16), (40, 2, 32), (64, 1, 256)])
def test_weights_against_float64(dtype, hd, H, kv, page):
    torch = torch_cuda()
    c = Case(hd + H + page, dtype, hd, H, kv, page, [1, 0, 2, 31, 33, 64, 127, 129, 257, 300, 513, 1100])
    total = torch.full_like(c.weight, -7.0)
    total.copy_(c.weight)
    got = c.run(weight_out=total)
    c.check(got, total)
    assert np.array_equal(host(c.weight), c.w64)
    again = c.run()                                          # in place
    assert np.array_equal(host(c.weight), host(total)) and np.array_equal(host(again[0]), host(got[0]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_rows_and_totals_with_columns_to_spare(dtype):
    torch_cuda()
    c = Case(9, dtype, 128, 8, 2, 16, [9011, 3, 2500, 0, 256 * 9], extra=37)
    got = c.run()
    c.check(got, c.weight)


def test_what_lies_behind_stays():
    """Totals of another tensor: only the row's keys are written."""
    torch = torch_cuda()
    c = Case(10, "bf16", 64, 4, 2, 16, [40, 0, 200])
    total = torch.full((3, 2, c.cap + 5), -7.0, device="cuda")
    c.run(weight_out=total)
    for r, n in enumerate(c.lens):
        assert (total[r, :, n:] == -7.0).all() and (total[r, :, :n] >= 0).all()


def test_missing_pages_lengths_and_sequences_of_weights():
    torch_cuda()
    c = Case(11, "bf16", 64, 8, 2, 16, [300, 300, 300, 40, 20])
    t, n = c.table.copy(), len(c.k64)
    t[0, :8] = -1
    t[1, 1::2] = n
    t[3, :] = -1
    total = c.weight.clone()
    c.check(c.run(table=t, weight_out=total), total, table=t)
    seq, lens = np.array([4, 7, -1, 0, 2]), np.array([2 ** 31 - 1, 5, 6, -9, 299])
    total = c.weight.clone()
    c.check(c.run(seq=seq, lens=lens, max_len=250, weight_out=total), total, seq=seq, lens=lens, max_len=250)
    total = c.weight.clone()
    c.check(c.run(max_len=0, weight_out=total), total, max_len=0)
    for scale in (0.7, -0.3, 0.0):
        total = c.weight.clone()
        c.check(c.run(scale=scale, weight_out=total), total, scale=scale)


def test_the_output_is_the_attentions():
    """weigh and attention differ in the order of sums alone."""
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    c = Case(12, "f32", 64, 8, 2, 16, [300, 1, 777])
    got = c.run()
    want = paged.attention(c.q, c.k, c.v, ints(c.table), ints(c.lens), return_lse=True)
    tol = 2 * span_bounds(1000, np.abs(host(want[0])).max(), np.full((1,), 40.0), 0.0, np.zeros(1), 64, "f32")[0]
    assert (np.abs(host(got[0]) - host(want[0])) <= tol.max()).all()


@pytest.mark.parametrize("cap,lens", [(1, [1, 0]), (50, [50, 49, 7]), (300, [300, 256, 257, 1]), (5000, [5000, 4097, 2500, 300])])
@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 0), (1, 1, 0), (2, 1, 1), (40, 4, 10), (256, 0, 100), (1999, 3, 501),
                                                 (6000, 1, 1)])
def test_evictions(cap, lens, budget, sinks, recent):
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(cap + budget)
    w = torch.from_numpy((rng.random((len(lens), 3, cap)) ** 4).astype(np.float32)).cuda()
    w[:, 1] = (w[:, 1] * 8).floor() / 8                      # many equal ones
    w[:, 2] = 0
    want = ref.evict(host(w), lens, budget, sinks, recent)
    out = torch.full_like(w, 7.0)
    got = paged.evict(w, ints(lens), budget, sinks=sinks, recent=recent, weight_out=out)
    assert np.array_equal(host(got[0]), want[0]) and np.array_equal(host(got[1]), want[1])
    assert np.array_equal(host(out), want[2])
    got = paged.evict(w, ints(lens), budget, sinks=sinks, recent=recent)      # in place
    assert np.array_equal(host(got[0]), want[0]) and np.array_equal(host(w), want[2])


def test_weights_that_are_not_finite_and_lengths_out_of_range():
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(3)
    w = torch.from_numpy(rng.standard_normal((4, 2, 700)).astype(np.float32)).cuda()
    w[:, :, 100] = float("nan")
    w[:, :, 90:95] = float("inf")
    w[:, 0, 5:60] = float("-inf")
    w[:, 1, 200:400:2] = -0.0
    w[:, 1, 201:400:2] = 0.0
    lens = [-3, 2 ** 31 - 1, 650, 8]
    for budget in (5, 400, 690):
        want = ref.evict(host(w), lens, budget, 2, 3)
        out = torch.empty_like(w)
        got = paged.evict(w, ints(lens), budget, sinks=2, recent=3, weight_out=out)
        assert np.array_equal(host(got[0]), want[0]) and np.array_equal(host(got[1]), want[1])
        assert np.array_equal(host(out), want[2], equal_nan=True)


@pytest.mark.parametrize("cap,lens,budget", [(40000, [40000, 16385, 100], 9001), (20000, [16384, 20000], 16384)])
def test_long_evictions(cap, lens, budget):
    """More keys than a workgroup holds at once, in place and not."""
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(cap)
    w = torch.from_numpy((rng.random((len(lens), 2, cap)) ** 4).astype(np.float32)).cuda()
    w[:, 1] = (w[:, 1] * 64).floor()
    want = ref.evict(host(w), lens, budget, 5, 77)
    out = torch.full_like(w, 7.0)
    got = paged.evict(w, ints(lens), budget, sinks=5, recent=77, weight_out=out)
    assert np.array_equal(host(got[0]), want[0]) and np.array_equal(host(got[1]), want[1])
    assert np.array_equal(host(out), want[2])
    paged.evict(w, ints(lens), budget, sinks=5, recent=77)
    assert np.array_equal(host(w), want[2])
