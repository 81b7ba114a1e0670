"""GPU: page bounds over a cache whose tokens come by drafted trees: after accept
the moved tokens' pages have the bounds of what they hold, and attention over
chosen pages is the definition's."""
import numpy as np
import pytest

from oracle import trees
from tests.gpu_common import torch_cuda
from tests.paged_common import host, ints
from tests.trees_common import check

pytestmark = pytest.mark.gpu

LAYERS, KV, H, HD, PS, S, T = 2, 2, 4, 32, 4, 3, 9


def test_bounds_after_accepted_paths():
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    cache = paged.PagedCache(LAYERS, KV, HD, PS, 60, S, 18, dtype=torch.float32, bounds=True)
    g = torch.Generator(device="cuda").manual_seed(3)
    rng = np.random.default_rng(3)
    draw = lambda heads: torch.randn((S * T, heads, HD), generator=g, device="cuda")
    seq = ints(np.repeat(np.arange(S), T))
    moved = 0
    for step in range(10):
        n_draft = np.array([T, rng.integers(0, T + 1), T - step % 3])
        before = cache.lens.clone()
        place = cache.reserve(ints(n_draft)).places(T).flatten()
        for layer in range(LAYERS):
            k = draw(KV)
            k[T // 2:] *= 10.0                               # rejected tokens widen a page's bounds
            cache.append(layer, place, draw(H), k, draw(KV), seq=seq)
            cache.update_bounds(layer, n_new=T)
        count = np.array([rng.integers(0, n + 1) for n in n_draft])
        path = np.full((S, T), -1)
        for s in range(S):
            path[s, :count[s]] = np.sort(rng.permutation(n_draft[s])[:count[s]])
            moved += int((path[s, :count[s]] != np.arange(count[s])).sum())
        cache.accept(before, ints(path), ints(count))
        assert np.array_equal(host(cache.lens), host(before) + count)
        table, lens = host(cache.table), host(cache.lens)
        used = table[table >= 0]
        for layer in range(LAYERS):
            cache.update_bounds(layer, n_new=T)
            want = trees.page_bounds(host(cache.k[layer]), table, lens, 1 << 30, np.zeros((60, KV, 2, HD)))
            assert np.array_equal(host(cache.bounds[layer])[used], want[used])
            q = draw(H)[:S].contiguous()
            got = cache.sparse_attention(layer, q, 5, sinks=1, recent=2, return_lse=True)
            columns = trees.select_pages(host(q), want, table, lens, PS, 5, 1, 2)
            out = trees.attend(host(q), host(cache.k[layer]), host(cache.v[layer]), trees.row_places(table, 60, PS, lens, columns))
            check([host(t) for t in got], out, 72, HD, "f32")
    assert moved > 20
