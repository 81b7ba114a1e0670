"""GPU: attention of one new token over a paged cache against float64, over
page sizes, lengths at every tile and split edge, head layouts, windows,
missing pages, groups of rows that share pages, strides, and non-finite values
where nothing looks."""
import numpy as np
import pytest

from oracle import paged as ref
from tests.gpu_common import torch_cuda
from tests.paged_common import attention_bounds, dtype_of, host, ints, normal, random_table

pytestmark = pytest.mark.gpu

EDGES = [1, 0, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 511, 512, 513, 769]


class Case:
    def __init__(self, seed, dtype, hd, H, kv, page, lens, q_scale=1.5):
        rng = np.random.default_rng(seed)
        self.rng, self.dtype, self.hd, self.page, self.lens = rng, dtype, hd, page, np.array(lens)
        self.table, n = random_table(rng, lens, page)
        self.k, self.k64 = normal(rng, (n, kv, page, hd), dtype)
        self.v, self.v64 = normal(rng, (n, kv, page, hd), dtype)
        self.q, self.q64 = normal(rng, (len(lens), H, hd), dtype, q_scale)

    def run(self, **kw):
        from paper_2606_29223_amd import paged
        lens = kw.pop("lens", self.lens)
        table = kw.pop("table", self.table)
        return paged.attention(kw.pop("q", self.q), self.k, self.v, ints(table), ints(lens), return_lse=True, **kw)

    def check(self, got, **kw):
        seq = kw.pop("rows_seq", None)
        out, lse, spread, size = ref.attention(kw.pop("q64", self.q64), self.k64, self.v64, kw.pop("table", self.table),
                                               kw.pop("lens", self.lens), seq=seq, **kw)
        tol, ltol = attention_bounds(self.q64, spread, size, out, lse, self.hd, self.dtype)
        g, l = host(got[0]), host(got[1])
        assert np.array_equal(np.isneginf(l), np.isneginf(lse))
        assert (np.abs(g - out) <= tol).all(), np.max(np.abs(g - out) / tol)
        ok = np.isfinite(lse)
        assert (np.abs(l[ok] - lse[ok]) <= ltol[ok]).all(), np.max(np.abs(l[ok] - lse[ok]) / ltol[ok])
        return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("H,kv,page", [(4, 4, 1), (6, 2, 8), (16, 1, 16), (10, 5, 64), (40, 2, 32), (64, 1, 256),
                                       (21, 3, 1024)])
def test_every_edge_against_float64(dtype, hd, H, kv, page):
    torch_cuda()
    c = Case(hd + H + page, dtype, hd, H, kv, page, EDGES)
    got = c.run()
    c.check(got)
    again = c.run(max_len=769)
    assert all(np.array_equal(host(a), host(b)) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 5, 64, 200, 256, 300, 100000])
def test_windows(dtype, window):
    torch_cuda()
    c = Case(window, dtype, 64, 8, 2, 16, EDGES)
    c.check(c.run(window=window), window=window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_rows(dtype):
    """Enough splits for a full join, rows of very different lengths."""
    torch_cuda()
    c = Case(9, dtype, 128, 8, 2, 16, [20011, 3, 9000, 0, 256 * 33])
    c.check(c.run())
    c.check(c.run(window=5000), window=5000)


def test_missing_pages_and_impossible_ones():
    """Pages that are -1 or no page at all are not attended to, at the front
    (slid out of a window), in the middle and behind; a row may be left with
    none."""
    torch_cuda()
    c = Case(21, "bf16", 64, 8, 2, 16, [700, 700, 700, 300, 40])
    t, n = c.table.copy(), len(c.k64)
    t[0, :20] = -1
    t[1, 3::2] = n
    t[2, 16:32] = 2 ** 31 - 1
    t[2, 0] = -2 ** 31
    t[3, :] = -1
    t[4, 1:] = n + 7
    c.check(c.run(table=t), table=t)


def test_lengths_and_sequences_out_of_range():
    """Negative lengths, lengths past max_len and past the table, sequences
    outside the table: clamped, or an empty row."""
    torch_cuda()
    c = Case(22, "bf16", 64, 4, 2, 16, [300, 300, 300, 300, 300, 300])
    lens = np.array([-3, 2 ** 31 - 1, 299, 300, -2 ** 31, 17])
    c.check(c.run(lens=lens, max_len=250), lens=lens, max_len=250)
    c.check(c.run(lens=lens), lens=lens)
    c.check(c.run(lens=lens, max_len=0), lens=lens, max_len=0)
    seq = np.array([0, 5, -1, 6, 2 ** 31 - 1, 2])
    c.check(c.run(seq=ints(seq)), rows_seq=seq)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_non_finite_values_where_nothing_looks(dtype):
    """NaN and infinities in unwritten slots, unused pages and keys before the
    window change no bit."""
    torch = torch_cuda()
    c = Case(23, dtype, 64, 8, 2, 16, [1, 5, 70, 250, 300])
    want = [host(t) for t in c.run(window=40)]
    used = np.zeros(c.k64.shape[:1] + (16,), bool)
    for s, n in enumerate(c.lens):
        for j in range(max(0, n - 40), n):
            used[ref.page_of(c.table, len(c.k64), 16, s, j)] = True
    hide = torch.from_numpy(~used).cuda()[:, None, :, None]
    for bad in (float("nan"), float("inf"), float("-inf"), 3e38):
        c.k.masked_fill_(hide, bad)
        c.v.masked_fill_(hide, bad)
        got = [host(t) for t in c.run(window=40)]
        assert all(np.array_equal(a, b) for a, b in zip(got, want)), bad


def test_large_scores_and_equal_keys():
    """One key far above the rest, all keys equal, scores of +-2000."""
    torch = torch_cuda()
    c = Case(24, "f32", 64, 4, 4, 16, [600, 600, 65], q_scale=200.0)
    c.check(c.run())
    c.k.copy_(c.k[:1, :, :1].expand_as(c.k))
    c.k64 = host(c.k)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [2, 3, 8])
@pytest.mark.parametrize("H,kv,hd", [(8, 2, 128), (4, 4, 64), (40, 2, 32)])
def test_rows_that_share_pages_keep_their_bits(dtype, group, H, kv, hd):
    """Beams with common leading pages, in groups that end anywhere, give the
    bits of single rows: shared for less than a split, for several, wholly,
    not at all, with different lengths, an empty row and a missing page."""
    torch_cuda()
    lens = [900, 900, 901, 700, 700, 200, 64, 0, 1300, 1300, 1290, 1300, 5, 5]
    c = Case(group + H, dtype, hd, H, kv, 16, lens)
    t = c.table
    t[1, :40] = t[0, :40]
    t[2, :33] = t[0, :33]
    t[4, :] = t[3, :]
    t[9, :64], t[10, :70], t[11, :81] = t[8, :64], t[8, :70], t[8, :81]
    t[12, 0] = t[13, 0]
    t[8, 5] = t[9, 5] = t[10, 5] = t[11, 5] = -1
    alone = c.run()
    c.check(alone)
    for kw in (dict(), dict(window=777)):
        a, b = c.run(group=1, **kw), c.run(group=group, **kw)
        assert all(np.array_equal(host(x), host(y)) for x, y in zip(a, b)), kw


def test_a_row_has_its_own_bits():
    """Whichever rows share the call, whatever max_len says."""
    torch_cuda()
    c = Case(31, "bf16", 128, 32, 8, 16, [5, 700, 2100, 64, 3000, 1])
    want = [host(t) for t in c.run()]
    for rows in ([4], [1, 1, 2], list(range(5, -1, -1))):
        seq = np.array(rows)
        got = c.run(q=c.q[rows], lens=c.lens[rows], seq=ints(seq), max_len=int(c.lens[rows].max()) + 900)
        assert all(np.array_equal(host(g), w[rows]) for g, w in zip(got, want))


def test_more_rows_than_a_launch_takes():
    torch_cuda()
    rows = 2100
    lens = np.arange(rows) % 97
    c = Case(32, "bf16", 32, 2, 1, 8, lens)
    c.check(c.run())
    c.check(c.run(group=4))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_queries_and_outputs(dtype):
    torch = torch_cuda()
    c = Case(33, dtype, 64, 6, 2, 16, [300, 65, 0])
    want, _ = c.run()
    fused = torch.zeros((3, 10, 64), dtype=c.q.dtype, device="cuda")
    fused[:, 1:7] = c.q
    out = torch.full((3, 12, 64), 5.0, dtype=c.q.dtype, device="cuda")
    got, _ = c.run(q=fused[:, 1:7], out=out[:, ::2])
    assert torch.equal(got, want) and (out[:, 1::2] == 5).all()
    flat = torch.zeros(3 * 6 * 64 + 3, dtype=c.q.dtype, device="cuda")
    odd, odd_out = flat[3:].view(3, 6, 64), torch.zeros(3 * 6 * 64 + 1, dtype=c.q.dtype, device="cuda")[1:].view(3, 6, 64)
    odd.copy_(c.q)
    got, _ = c.run(q=odd, out=odd_out)
    assert torch.equal(got, want)


def test_offsets_past_32_bits():
    """A layer of more than 2^32 bytes and 2^31 elements, its last pages used."""
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    n_pages, kv, page, hd = 2 ** 31 // (8 * 16 * 128) + 700, 8, 16, 128
    k = torch.empty((n_pages, kv, page, hd), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    rng = np.random.default_rng(34)
    table = np.stack([np.arange(n_pages - 20, n_pages), np.arange(20)])
    for i in list(table.flatten()):
        k[i].normal_()
        v[i].normal_()
    q, q64 = normal(rng, (2, 16, hd), "bf16")
    lens = np.array([311, 320])
    got = paged.attention(q, k, v, ints(table), ints(lens), return_lse=True)
    ids = torch.from_numpy(table.flatten()).cuda()
    small = np.arange(40).reshape(2, 20)
    out, lse, spread, size = ref.attention(q64, host(k[ids]), host(v[ids]), small, lens)
    tol, ltol = attention_bounds(q64, spread, size, out, lse, hd, "bf16")
    assert (np.abs(host(got[0]) - out) <= tol).all() and (np.abs(host(got[1]) - lse) <= ltol).all()
    x, x64 = normal(rng, (2, 8, hd), "bf16")              # and the write lands there too
    paged.append(k, v, ints(table), ints([311, 312]), x, x)
    assert torch.equal(v[n_pages - 1, :, 7], x[0]) and torch.equal(k[19, :, 8], x[1])


@pytest.mark.parametrize("dtype,group", [("bf16", 1), ("bf16", 4), ("f32", 4)])
def test_a_captured_call_follows_lengths_and_tables(dtype, group):
    """Captured once, replayed with other lengths, other tables and other
    queries: every replay has the bits of an eager call on them."""
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    c = Case(41, dtype, 128, 8, 2, 16, [900, 900, 900, 900, 2500, 2400, 700, 0])
    t = c.table.copy()
    t[1, :50] = t[2, :40].tolist() + t[1, 40:50].tolist()
    table, lens, q = ints(t), ints(c.lens), c.q.clone()
    run = lambda: paged.attention(q, c.k, c.v, table, lens, max_len=2560, group=group, window=1500, return_lse=True)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = run()
    for i in range(5):
        new = c.rng.permutation(8)
        table.copy_(ints(t[new]))
        lens.copy_(ints(np.maximum(c.lens[new] - 37 * i, 0)))
        q.copy_(c.q[torch.from_numpy(c.rng.permutation(8)).cuda()])
        want = run()
        graph.replay()
        if i % 2:
            torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]), i


def test_calls_that_overlap_on_two_streams():
    torch = torch_cuda()
    cases = [Case(s, "bf16", 128, 16, 4, 16, [3000, 1200, 4000, 65]) for s in (51, 52)]
    want = [c.run() for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(6):
        got = []
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                got.append(c.run())
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])
