"""GPU: beam selection's totals follow from the logits alone, not from where the
rows begin in memory: beams with the same logits and scores tie exactly, and go
by beam and token."""
import numpy as np
import pytest

from oracle import paged as ref
from tests.gpu_common import torch_cuda
from tests.paged_common import dtype_of, host

pytestmark = pytest.mark.gpu


def _row(rng, vocab, scale, dtype):
    torch = torch_cuda()
    return torch.from_numpy((scale * rng.standard_normal((1, vocab))).astype(np.float32)).to(dtype_of(dtype)).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [301, 4099, 32001, 65537])
@pytest.mark.parametrize("scale", [1.0, 3.0, 10.0])
def test_equal_beams_tie_at_any_alignment(dtype, vocab, scale):
    """Eight beams of an odd vocabulary: each row begins elsewhere in 16 bytes."""
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(vocab)
    requests, beams = 3, 8
    rows = torch.cat([_row(rng, vocab, scale, dtype).expand(beams, vocab) for _ in range(requests)]).contiguous()
    scores = np.full((requests, beams), -1.25, np.float32)
    for n in (beams, 20):
        got = paged.beam_select(rows, torch.from_numpy(scores).cuda(), n_out=n)
        want = ref.beam_select(host(rows), scores, n)
        assert np.array_equal(host(got[0]), want[0]) and np.array_equal(host(got[1]), want[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [77, 2049, 9000, 40001])
def test_a_row_has_the_same_bits_anywhere(dtype, vocab):
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(vocab)
    row, score = _row(rng, vocab, 4.0, dtype), torch.zeros((1, 1), device="cuda")
    flat = torch.full((vocab + 16,), float("nan"), dtype=row.dtype, device="cuda")        # nothing beside the row is read
    want = None
    for off in range(9):
        view = flat[off:off + vocab].view(1, vocab)
        view.copy_(row)
        got = [host(t) for t in paged.beam_select(view, score, n_out=12)]
        view.fill_(float("nan"))
        want = want or got
        assert all(np.array_equal(a, b) for a, b in zip(got, want)), off
