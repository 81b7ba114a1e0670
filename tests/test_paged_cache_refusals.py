"""PagedCache refuses calls whose results would not be the caller's tensors or the
caller's rows, before anything is launched."""
import pytest

torch = pytest.importorskip("torch")

from paper_2606_29223_amd import dexlib, paged  # noqa: E402

LAYERS, KV, HD, PS, SEQS, WIDTH = 2, 2, 32, 4, 3, 5


def cache(**kw):
    return paged.PagedCache(LAYERS, KV, HD, PS, 8, SEQS, WIDTH, device="cpu", **kw)


@pytest.mark.parametrize("view", [
    lambda n: torch.zeros((SEQS, LAYERS, KV, n)).transpose(0, 1),
    lambda n: torch.zeros((LAYERS, SEQS, n, KV)).transpose(2, 3),
    lambda n: torch.zeros((LAYERS, SEQS, KV, n + 4))[..., :n],
    lambda n: torch.zeros((LAYERS, SEQS + 1, KV, n))[:, 1:],
    lambda n: torch.zeros((LAYERS, 1, KV, n)).expand(LAYERS, SEQS, KV, n)])
def test_evict_refuses_weights_that_it_could_not_cut_in_place(view):
    """Flattened over layers and sequences these are copies: the caller's totals
    would stay as they were."""
    weight = view(PS * WIDTH)
    assert weight.shape == (LAYERS, SEQS, KV, PS * WIDTH)
    with pytest.raises(dexlib.DexError, match="contiguous"):
        cache().evict(weight, 4)


def test_rows_of_other_sequences_come_with_their_lengths():
    """cache.lens[r] is sequence r's length, not that of sequence seq[r]."""
    seq, q = torch.tensor([2, 0, 1], dtype=torch.int32), torch.zeros((SEQS, 4, HD))
    c = cache(bounds=True)
    for call in (lambda: c.sparse_attention(0, q, 2, seq=seq), lambda: c.weigh(0, q, torch.zeros((SEQS, KV, PS * WIDTH)), seq=seq)):
        with pytest.raises(dexlib.DexError, match="lens"):
            call()


def test_evict_refuses_weights_narrower_than_the_sequences_may_be():
    """Keys without a weight, the most recent ones, would be dropped."""
    narrow = torch.zeros((LAYERS, SEQS, KV, PS * WIDTH - 1))
    for max_len in (None, PS * WIDTH, 1 << 40):
        with pytest.raises(dexlib.DexError, match="columns"):
            cache().evict(narrow, 4, max_len=max_len)
    with pytest.raises(dexlib.DexError, match="max_len"):
        cache().evict(narrow, 4, max_len=-1)
    for weight, max_len in ((narrow, PS * WIDTH - 1), (narrow, 3), (torch.zeros((LAYERS, SEQS, KV, PS * WIDTH)), None)):
        with pytest.raises(dexlib.DexError, match="GPU"):     # wide enough: refused for where it is alone
            cache().evict(weight, 4, max_len=max_len)
