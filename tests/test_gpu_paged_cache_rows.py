"""GPU: PagedCache's attention over chosen pages and its weights, of rows that are
other sequences than their number, against float64."""
import numpy as np
import pytest

from oracle import trees as ref
from tests.gpu_common import torch_cuda
from tests.paged_common import host, ints
from tests.trees_common import check

pytestmark = pytest.mark.gpu

KV, H, HD, PS = 2, 4, 32, 4
LENS = [30, 9, 0, 47]
SEQ = np.array([3, 0, 3, 1, 2, 1, -1])
ROW_LENS = np.array([47, 30, 21, 9, 0, 5, 12])


def _cache(seed):
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    cache = paged.PagedCache(1, KV, HD, PS, 40, 4, 20, dtype=torch.float32, bounds=True)
    cache.reserve(ints(LENS))
    g = torch.Generator(device="cuda").manual_seed(seed)
    for x in (cache.k, cache.v):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
    cache.update_bounds(0)
    return cache, torch.randn((len(SEQ), H, HD), generator=g, device="cuda")


@pytest.mark.parametrize("max_len", [None, 47, 48, 30])
def test_chosen_pages_of_other_sequences(max_len):
    torch_cuda()
    cache, q = _cache(1)
    table, k, v = host(cache.table), host(cache.k[0]), host(cache.v[0])
    seen = np.minimum(ROW_LENS, 80 if max_len is None else max_len)
    got = cache.sparse_attention(0, q, 4, sinks=1, recent=1, lens=ints(seen), seq=ints(SEQ), max_len=max_len, return_lse=True)
    columns = np.full((len(SEQ), KV, 4), -1)
    for r, s in enumerate(SEQ):
        if 0 <= s < 4:
            columns[r] = ref.select_pages(host(q)[r:r + 1], host(cache.bounds[0]), table[s:s + 1], seen[r:r + 1], PS, 4, 1, 1)[0]
    want = ref.attend(host(q), k, v, ref.row_places(table, 40, PS, seen, columns, seq=SEQ))
    check([host(t) for t in got], want, 80, HD, "f32")
    same = cache.sparse_attention(0, q[:4], 4, max_len=max_len, lens=ints(np.minimum(LENS, seen.max())))
    assert (host(same)[2] == 0).all()


def test_weights_of_other_sequences():
    torch = torch_cuda()
    cache, q = _cache(2)
    weight = torch.ones((len(SEQ), KV, 80), device="cuda")
    got = cache.weigh(0, q, weight, lens=ints(ROW_LENS), seq=ints(SEQ), return_lse=True)
    want = ref.attend(host(q), host(cache.k[0]), host(cache.v[0]), ref.row_places(host(cache.table), 40, PS, ROW_LENS, seq=SEQ))
    check([host(t) for t in got], want, 80, HD, "f32")
    for r, s in enumerate(SEQ):
        n = int(ROW_LENS[r]) if 0 <= s < 4 else 0
        total = host(weight)[r]
        # every head's weights come to one; each is off by 2^-20 at most here (scores up to 30), the total by its rounding
        assert np.allclose(total[:, :n].sum(1) - n, H // KV if n else 0, atol=(n + 2) * 2.0 ** -20)
        assert (total[:, n:] == 1).all()
