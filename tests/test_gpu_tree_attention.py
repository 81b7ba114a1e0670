"""GPU: attention of trees of drafted tokens over a paged cache against float64,
over head layouts, page sizes, lengths and trees at every tile and split edge,
any masks, missing pages, strides, and non-finite values that some rows see and
others do not."""
import numpy as np
import pytest

from oracle import trees as ref
from tests.gpu_common import torch_cuda
from tests.paged_common import host, ints, normal, random_table
from tests.trees_common import check, random_tree

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, seed, dtype, hd, H, kv, page, lens, draft, q_scale=1.5, drafts=None):
        rng = np.random.default_rng(seed)
        self.rng, self.dtype, self.hd, self.page, self.draft = rng, dtype, hd, page, draft
        self.lens = np.array(lens)
        self.drafts = None if drafts is None else np.array(drafts)
        d = np.full(len(lens), draft) if drafts is None else self.drafts
        self.table, n = random_table(rng, self.lens + d, page)
        self.k, self.k64 = normal(rng, (n, kv, page, hd), dtype)
        self.v, self.v64 = normal(rng, (n, kv, page, hd), dtype)
        self.q, self.q64 = normal(rng, (len(lens) * draft, H, hd), dtype, q_scale)
        self.seen, _ = ref.tree_mask(np.stack([random_tree(rng, draft) for _ in lens]))

    def run(self, **kw):
        from paper_2606_29223_amd import paged
        torch = torch_cuda()
        seen = kw.pop("seen", self.seen)
        mask = torch.from_numpy(ref.words(seen)).cuda()
        nd = kw.pop("drafts", self.drafts)
        return paged.tree_attention(kw.pop("q", self.q), self.k, self.v, ints(kw.pop("table", self.table)),
                                    ints(kw.pop("lens", self.lens)), mask, n_draft=None if nd is None else ints(nd),
                                    return_lse=True, **kw)

    def want(self, **kw):
        places = ref.tree_places(kw.pop("table", self.table), len(self.k64), self.page, kw.pop("lens", self.lens),
                                 kw.pop("seen", self.seen), kw.pop("drafts", self.drafts), kw.pop("seq", None),
                                 kw.pop("max_len", None))
        return ref.attend(self.q64, self.k64, self.v64, places, **kw)

    def check(self, got, **kw):
        check([host(t) for t in got], self.want(**kw), int(max(self.lens.max(), 0)) + self.draft, self.hd, self.dtype)


LAYOUTS = [(4, 4, 1), (6, 2, 8), (16, 1, 16), (10, 5, 64), (64, 1, 256)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("H,kv,page", LAYOUTS)
def test_short_sequences_against_float64(dtype, hd, H, kv, page):
    torch_cuda()
    for draft, lens in ((1, [0, 1, 31, 32, 33, 64, 127, 129, 300]), (5, [0, 27, 28, 60, 123, 250])):
        c = Case(hd + H + page + draft, dtype, hd, H, kv, page, lens, draft)
        c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("draft", [2, 4, 8, 16, 17, 31, 33, 63, 64, 65, 100, 128, 129, 200, 256])
def test_every_size_of_tree(dtype, draft):
    """Four heads a kv head: 8 to 1024 columns of the products."""
    torch_cuda()
    c = Case(draft, dtype, 64, 4, 1, 16, [0, 3, 70, 261], draft)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,draft", [(128, 3), (128, 12), (128, 40), (32, 70)])
def test_long_sequences(dtype, hd, draft):
    """Enough splits for the join, of very different lengths, ragged trees."""
    torch_cuda()
    c = Case(9, dtype, hd, 4, 2, 16, [7011, 3, 2900, 0, 1024], draft, drafts=[draft, 1, draft - 1, draft, 2])
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,draft", [(128, 3), (64, 13), (128, 30)])
@pytest.mark.parametrize("page", [1, 2])
def test_more_pages_than_a_wave_holds(dtype, hd, draft, page):
    """64 columns of a table are looked at at once: keys on both sides of that, and
    of the splits, some of their pages missing."""
    torch_cuda()
    c = Case(hd + page, dtype, hd, 8, 2, page, [0, 61, 63, 64, 65, 127, 129, 703, 2000], draft)
    t = c.table.copy()
    t[3:, 5::7] = -1
    c.check(c.run(table=t), table=t)


def many_wide(dtype, hd, page):
    """Trees of 20 with four heads a kv head, 80 columns, in enough (tree, kv head)
    pairs that a wave takes two blocks of columns."""
    lens = [0, 1, 30, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 257, 300, 511, 1500, 3100, 12]
    return Case(hd + page, dtype, hd, 8, 2, page, lens, 20, drafts=[20, 1, 0, 19] * 4 + [20, 20, 7, 20])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,page", [(32, 4), (64, 1), (64, 16), (128, 2), (128, 64)])
def test_many_wide_trees(dtype, hd, page):
    torch_cuda()
    c = many_wide(dtype, hd, page)
    c.check(c.run())
    t = c.table.copy()
    t[10:, 3::5] = -1
    c.check(c.run(table=t), table=t)
    seq = np.array([19, 18, 17, -1, 20] + list(range(15)))
    lens = np.concatenate((c.lens[19:16:-1], [40, 40], c.lens[:15]))
    drafts = np.concatenate((c.drafts[19:16:-1], [20, 20], c.drafts[:15]))
    c.check(c.run(seq=ints(seq), lens=lens, drafts=drafts), seq=seq, lens=lens, drafts=drafts)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_wide_trees_with_values_that_only_some_rows_see(dtype):
    torch_cuda()
    c = many_wide(dtype, 64, 16)
    c.seen[:] = np.eye(20, dtype=bool)
    c.seen[:, 10:, 1] = True
    clean = [host(t) for t in c.run()]
    sees = np.zeros((20, 20), bool)
    for b, n in enumerate(c.lens):
        if c.drafts[b] > 1:
            c.v[int(c.table[b, (n + 1) // 16]), :, (n + 1) % 16, 7] = float("-inf")
            sees[b] = c.seen[b, :, 1] & (np.arange(20) < c.drafts[b])
    got = [host(t) for t in c.run()]
    sees = sees.reshape(-1)
    assert np.isneginf(got[0][sees][..., 7]).all() and np.array_equal(got[0][~sees], clean[0][~sees])
    assert np.array_equal(np.delete(got[0], 7, 2), np.delete(clean[0], 7, 2)) and np.array_equal(got[1], clean[1])


def test_drafts_out_of_range_and_sequences_that_are_none():
    """Rows from n_draft on get zeros and -inf; n_draft, lens and sequences out
    of range are clamped or leave the tree empty."""
    torch_cuda()
    c = Case(3, "bf16", 64, 8, 2, 8, [50, 60, 70, 80, 90], 7)
    nd = np.array([0, -5, 99, 3, 2 ** 31 - 1])
    got = c.run(drafts=nd)
    c.check(got, drafts=nd)
    assert (host(got[0])[:14] == 0).all() and np.isneginf(host(got[1])[:14]).all()
    lens = np.array([-3, 2 ** 31 - 1, 10, 79, -2 ** 31])
    c.check(c.run(lens=lens, max_len=64), lens=lens, max_len=64)
    c.check(c.run(lens=lens), lens=lens)
    c.check(c.run(max_len=0), max_len=0)
    seq = np.array([4, 5, -1, 0, 2 ** 31 - 1])
    c.check(c.run(seq=ints(seq)), seq=seq)


def test_any_mask():
    """Masks that are no tree: random bits, nothing at all, later nodes."""
    torch_cuda()
    for draft in (6, 64, 90):
        c = Case(draft, "bf16", 64, 4, 2, 16, [0, 5, 300], draft)
        seen = c.rng.random(c.seen.shape) < 0.3
        seen[:, 1] = False
        c.check(c.run(seen=seen), seen=seen)


def test_missing_pages():
    torch_cuda()
    c = Case(21, "bf16", 64, 8, 2, 16, [300, 300, 300, 40, 200], 9)
    t, n = c.table.copy(), len(c.k64)
    t[0, :8] = -1
    t[1, 3::2] = n
    t[2, 0] = -2 ** 31
    t[2, 18:] = 2 ** 31 - 1                                   # the drafted keys too
    t[3, :] = -1
    t[4, 12] = n + 7
    c.check(c.run(table=t), table=t)


@pytest.mark.parametrize("scale", [0.3, -0.2, 0.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales(dtype, scale):
    torch_cuda()
    c = Case(31, dtype, 32, 6, 3, 4, [0, 9, 150], 5)
    c.check(c.run(scale=scale), scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(dtype):
    """Scores whose references rise by far more than 2^8 along a row."""
    torch = torch_cuda()
    c = Case(32, dtype, 64, 4, 2, 16, [400, 33], 6, q_scale=40.0)
    ramp = torch.linspace(0.01, 3.0, c.k.shape[0], device="cuda")[:, None, None, None]
    c.k.mul_(ramp.to(c.k.dtype))
    c.k64 = host(c.k)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("draft", [3, 12, 20, 40])
def test_non_finite_keys_and_values_that_only_some_rows_see(dtype, draft):
    """A NaN or infinity at a drafted token reaches the rows that see it, as
    softmax has it, and changes no bit of the others; nor does anything behind
    the sequences or in other pages."""
    torch = torch_cuda()
    c = Case(draft, dtype, 64, 8, 2, 16, [40, 61, 0], draft)
    c.seen[:] = np.eye(draft, dtype=bool)                     # every node sees itself
    c.seen[:, draft // 2:, 0] = True                          # half of them the first
    clean = [host(t) for t in c.run()]
    used = np.zeros(c.k64.shape[:1] + (16,), bool)
    for b, n in enumerate(c.lens):
        for p in range(n + draft):
            used[c.table[b, p // 16], p % 16] = True
    hide = torch.from_numpy(~used).cuda()[:, None, :, None]
    for bad in (float("nan"), float("inf"), float("-inf")):
        c.k.masked_fill_(hide, bad)
        c.v.masked_fill_(hide, bad)
        assert all(np.array_equal(a, host(b)) for a, b in zip(clean, c.run())), bad
    for b, n in enumerate(c.lens):
        page, slot = int(c.table[b, n // 16]), n % 16
        old = c.v[page, :, slot].clone()
        for bad in (float("nan"), float("inf"), float("-inf")):
            c.v[page, :, slot, 5] = bad
            got = [host(t) for t in c.run()]
            rows = np.arange(b * draft, (b + 1) * draft)
            sees = c.seen[b, :, 0]
            g = got[0][rows]
            assert np.array_equal(g[~sees], clean[0][rows][~sees]), bad
            assert np.array_equal(np.delete(g, 5, 2), np.delete(clean[0][rows], 5, 2)), bad
            assert np.array_equal(g[sees][..., 5], np.full_like(g[sees][..., 5], bad), equal_nan=True), bad
            assert np.array_equal(got[1], clean[1])
        c.v[page, :, slot] = old
        old = c.k[page, :, slot].clone()
        c.k[page, :, slot, 2] = float("nan")
        g = host(c.run()[0])[rows]
        assert np.array_equal(g[~sees], clean[0][rows][~sees]) and np.isnan(g[sees]).all()
        c.k[page, :, slot] = old


@pytest.mark.parametrize("draft", [1, 6, 40])
def test_infinite_values_before_the_tree(draft):
    """Every row sees them: infinite of one sign, NaN for both."""
    torch_cuda()
    c = Case(draft, "bf16", 64, 8, 2, 16, [300, 90], draft)
    for b, at in ((0, 250), (1, 3)):
        c.v[int(c.table[b, at // 16]), :, at % 16, 4] = float("-inf")
        c.v[int(c.table[b, at // 16]), :, at % 16, 9] = float("inf")
        c.v[int(c.table[b, (at + 1) // 16]), :, (at + 1) % 16, 9] = float("-inf")
    got, clean = host(c.run()[0]), c.want()[0]
    assert np.isneginf(got[..., 4]).all() and np.isnan(got[..., 9]).all()
    assert np.isfinite(np.delete(got, (4, 9), 2)).all() and clean.shape == got.shape


def test_offsets_past_32_bits():
    """Pages behind more than 2^32 elements of a layer."""
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    c = Case(41, "bf16", 128, 4, 1, 1024, [1500, 40], 5)
    n = (1 << 32) // (1024 * 128) + 8
    k, v = (torch.empty((n, 1, 1024, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    far = np.where(c.table >= 0, c.table + n - len(c.k64), -1)
    k[n - len(c.k64):], v[n - len(c.k64):] = c.k, c.v
    want = [host(t) for t in c.run()]
    mask = torch.from_numpy(ref.words(c.seen)).cuda()
    got = paged.tree_attention(c.q, k, v, ints(far), ints(c.lens), mask, return_lse=True)
    assert all(np.array_equal(a, host(b)) for a, b in zip(want, got))
    # the same tokens moved, and their bounds
    bounds = paged.page_bounds(k, ints(far), ints(c.lens))
    near = paged.page_bounds(c.k, ints(c.table), ints(c.lens))
    assert torch.equal(bounds[n - len(c.k64):], near)
    index = ints(np.tile(np.arange(0, 1400, 2), (2, 1)))
    count = ints([700, 20])
    paged.keep(k[None], v[None], ints(far), index, count)
    paged.keep(c.k[None], c.v[None], ints(c.table), index, count)
    assert torch.equal(k[n - len(c.k64):], c.k) and torch.equal(v[n - len(c.k64):], c.v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_and_unaligned_queries_and_outputs(dtype):
    torch = torch_cuda()
    c = Case(5, dtype, 64, 6, 2, 8, [70, 130], 11)
    want = [host(t) for t in c.run()]
    n, H, hd = c.q.shape
    for pad, off in ((2 * H, 0), (1, 3), (0, 1)):
        x = torch.full((n, H + pad, hd + 7), 9.0, dtype=c.q.dtype, device="cuda")
        q = x[:, :H, off:off + hd]
        q.copy_(c.q)
        y = torch.full((n, H + pad, hd + 7), 9.0, dtype=c.q.dtype, device="cuda")
        out = y[:, :H, off:off + hd]
        got = c.run(q=q, out=out)
        assert got[0] is out and all(np.array_equal(a, host(b)) for a, b in zip(want, got))
        rest = y.clone()
        rest[:, :H, off:off + hd] = 9.0
        assert (rest == 9.0).all()
    heads_first = c.q.transpose(0, 1).contiguous().transpose(0, 1)
    assert all(np.array_equal(a, host(b)) for a, b in zip(want, c.run(q=heads_first)))


def test_trees_do_not_change_each_others_bits():
    """A tree alone, and beside others of other lengths: the same cut, the same
    bits (the number of trees decides the cut, so it stays)."""
    torch_cuda()
    c = Case(6, "bf16", 64, 4, 2, 16, [500, 900, 33], 5)
    want = host(c.run()[0])
    lens = np.array([1, 900, 600 - 5])
    lens[2] = 28
    got = host(c.run(lens=lens)[0])
    assert np.array_equal(want[5:10], got[5:10])
    again = host(c.run()[0])
    assert np.array_equal(want, again)


def test_no_trees():
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    c = Case(7, "bf16", 64, 4, 2, 16, [5], 3)
    none = torch.empty((0, 3, 1), dtype=torch.int64, device="cuda")
    out, lse = paged.tree_attention(c.q[:0], c.k, c.v, ints(c.table), ints([]), none, return_lse=True)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
