"""GPU: masks of trees, the accepted path, tokens moved inside their sequences
and pages given back, against the definitions: all whole numbers and copies."""
import numpy as np
import pytest

from oracle import trees as ref
from tests.gpu_common import torch_cuda
from tests.paged_common import dtype_of, host, ints, random_table
from tests.trees_common import random_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("draft", [1, 2, 31, 63, 64, 65, 127, 128, 129, 200, 256])
def test_masks_and_depths(draft):
    torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(draft)
    parent = np.stack([random_tree(rng, draft, roots=r) for r in (1, min(3, draft), 1)]
                      + [np.arange(draft) - 1, rng.integers(-5, draft + 5, draft)])
    mask, depth = paged.tree_mask(ints(parent))
    seen, want = ref.tree_mask(parent)
    assert np.array_equal(host(mask), ref.words(seen)) and np.array_equal(host(depth), want)


@pytest.mark.parametrize("draft", [1, 2, 7, 64, 65, 256])
@pytest.mark.parametrize("tokens", [1, 2, 5])
def test_accepted_paths(draft, tokens):
    """Few tokens make many nodes agree, several equally deep ones too."""
    torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(draft + tokens)
    n = 12
    parent = np.stack([random_tree(rng, draft, roots=min(draft, 1 + i % 3)) for i in range(n)])
    parent[0] = np.arange(draft) - 1
    token, target = rng.integers(0, tokens, (n, draft)), rng.integers(0, tokens, (n, draft))
    nd = rng.integers(-1, draft + 2, n)
    root = rng.integers(0, tokens, n)
    for a, b in ((None, None), (nd, None), (nd, root), (None, root)):
        got = paged.tree_accept(ints(parent), ints(token), ints(target), n_draft=None if a is None else ints(a),
                                root=None if b is None else ints(b))
        want = ref.tree_accept(parent, token, target, a, b)
        assert all(np.array_equal(host(x), y) for x, y in zip(got, want))


def pool(rng, shape, dtype):
    torch = torch_cuda()
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dtype_of(dtype)).cuda()


def rising(rng, n, most):
    """n numbers, each at least its place."""
    return np.maximum(np.sort(rng.permutation(most)[:n]), np.arange(n))


@pytest.mark.parametrize("dtype,hd,page", [("bf16", 128, 16), ("f32", 128, 1), ("bf16", 8, 4), ("bf16", 64, 256), ("f32", 36, 8),
                                           ("bf16", 520, 2)])
@pytest.mark.parametrize("lists", [2, 3, 4])
@pytest.mark.parametrize("away", [False, True])
def test_tokens_move(dtype, hd, page, lists, away):
    torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(hd + page + lists)
    layers, kv = 2, 3
    lens = np.array([700, 5, 0, 300])
    fresh = np.array([430, 60, 20, 300])
    table, used = random_table(rng, lens, page, 0)
    to, more = random_table(rng, fresh, page, 2)
    n_pages = used + more
    to = np.where(to >= 0, to + used, -1)
    shape = {2: (4, 400), 3: (4, kv, 400), 4: (layers, 4, kv, 400)}[lists]
    index = np.full(shape, -1)
    first = np.array([3, 0, 4, 150])
    count = np.array([400, 3, 7, 120])
    for at in np.ndindex(shape[:-1]):
        s = at[0] if lists < 4 else at[1]
        most = int(lens[s] - first[s])
        if most > 0:
            index[at][:min(count[s], most)] = rising(rng, min(count[s], most), most)
    index[..., 2] = -1                                       # a hole, and one past the table
    index[..., 1] = 2 ** 31 - 1
    if away:
        index[0, ..., 5:9] = index[0, ..., 5:6] // 2         # out of order, and twice the same
    k, v = pool(rng, (layers, n_pages, kv, page, hd), dtype), pool(rng, (layers, n_pages, kv, page, hd), dtype)
    lists_of = {2: lambda l, s, g: index[s], 3: lambda l, s, g: index[s, g], 4: lambda l, s, g: index[l, s, g]}[lists]
    want = ref.keep(host(k), host(v), table, lists_of, count, first, to if away else None)
    paged.keep(k, v, ints(table), ints(index), ints(count), first=ints(first), to=ints(to) if away else None)
    assert np.array_equal(host(k), want[0]) and np.array_equal(host(v), want[1])


def test_tokens_move_in_place_over_long_lists():
    """Several turns, whose sources lie among the places already written."""
    torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(0)
    lens = np.array([5000, 3000])
    table, n = random_table(rng, lens, 16)
    k, v = pool(rng, (1, n, 2, 16, 64), "bf16"), pool(rng, (1, n, 2, 16, 64), "bf16")
    index = np.full((2, 2, 4000), -1)
    for s in range(2):
        for g in range(2):
            m = int(lens[s]) * 4 // 5 - 7 * g
            index[s, g, :m] = rising(rng, m, int(lens[s]))
    index[0, 0, 100:140] = 4999                              # any order, as long as none lies before its place
    count = np.array([9000, 2000])
    want = ref.keep(host(k), host(v), table, lambda l, s, g: index[s, g], count)
    paged.keep(k, v, ints(table), ints(index), ints(count))
    assert np.array_equal(host(k), want[0]) and np.array_equal(host(v), want[1])


def test_counts_and_places_that_do_not_fit():
    """Negative counts and firsts, pages that are none: nothing is copied."""
    torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(1)
    table, n = random_table(rng, [64, 64, 64, 64], 8)
    table[2, 3:] = n + 1
    table[3, :2] = -1
    k, v = pool(rng, (2, n, 1, 8, 16), "f32"), pool(rng, (2, n, 1, 8, 16), "f32")
    index = np.tile(np.arange(20) * 3, (4, 1))
    count, first = np.array([-4, 20, 20, 20]), np.array([0, -1, 2, 2 ** 31 - 1])
    for f in (first, np.array([5, 2 ** 31 - 40, 2, 0])):
        want = ref.keep(host(k), host(v), table, lambda l, s, g: index[s], count, f)
        paged.keep(k, v, ints(table), ints(index), ints(count), first=ints(f))
        assert np.array_equal(host(k), want[0]) and np.array_equal(host(v), want[1])


@pytest.mark.parametrize("page", [1, 16, 1024])
@pytest.mark.parametrize("seqs,width", [(1, 1), (5, 40), (300, 70)])
def test_pages_given_back(page, seqs, width):
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(page + seqs)
    n = 9000
    table = rng.integers(-1, n, (seqs, width))
    table[0, -1] = n + 3
    ref_ = np.bincount(table[(table >= 0) & (table < n)], minlength=n) + rng.integers(0, 2, n)
    lens = rng.integers(-3, width * page + 20, seqs)
    lens[0] = 2 ** 31 - 1 if seqs > 1 else -2 ** 31
    want = ref.trim(table, ref_, lens, page)
    t, r = ints(table), ints(ref_)
    out = (torch.full_like(t, 77), torch.full_like(r, 77))
    got = paged.trim(t, r, ints(lens), page, out=out)
    assert got[0] is out[0] and np.array_equal(host(t), table) and np.array_equal(host(r), ref_)
    assert all(np.array_equal(host(a), b) for a, b in zip(got, want))
    got = paged.trim(t, r, ints(lens), page)
    assert got[0] is t and all(np.array_equal(host(a), b) for a, b in zip(got, want))
