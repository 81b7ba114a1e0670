"""GPU: beam selection against a float64 sort: parents, tokens and finished
marks exactly, scores to float rounding (the sum of exponentials is off by
about 2^-24 and the score is rounded once: 2^-22 of a few tens)."""
import math

import numpy as np
import pytest

from oracle import paged as ref
from tests.gpu_common import torch_cuda
from tests.paged_common import dtype_of, host

pytestmark = pytest.mark.gpu


def _run(logits, scores, n_out=None, done=None, eos=-1, x=None):
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    d = None if done is None else torch.from_numpy(done).cuda()
    got = paged.beam_select(logits, torch.from_numpy(scores.astype(np.float32)).cuda(), n_out=n_out, done=d, eos=eos)
    n = scores.shape[1] if n_out is None else n_out
    want = ref.beam_select(host(logits) if x is None else x, scores.astype(np.float32), n, done, eos)
    for name, a, b in zip(("parent", "token", "done"), (got[0], got[1], got[3]), (want[0], want[1], want[3])):
        assert np.array_equal(host(a), b), (name, host(a), b)
    a, b = host(got[2]), want[2]
    assert np.array_equal(np.isneginf(a), np.isneginf(b))
    ok = np.isfinite(b)
    assert (np.abs(a[ok] - b[ok]) <= 2.0 ** -22 * (np.abs(b[ok]) + 32)).all()
    return got


def _logits(rng, rows, vocab, dtype, scale=3.0):
    torch = torch_cuda()
    return torch.from_numpy((scale * rng.standard_normal((rows, vocab))).astype(np.float32)).to(dtype_of(dtype)).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("requests,beams,vocab,n_out", [(1, 1, 1, 1), (1, 4, 3, 12), (2, 3, 2048, 3), (1, 4, 32000, 4),
                                                        (3, 8, 5001, 16), (2, 64, 700, 64), (1, 2, 140001, 5),
                                                        (5, 5, 7, 10), (40, 2, 129, 64)])
def test_against_a_full_sort(dtype, requests, beams, vocab, n_out):
    rng = np.random.default_rng(vocab + beams)
    scores = -5 * rng.random((requests, beams))
    _run(_logits(rng, requests * beams, vocab, dtype), scores, n_out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ties_go_to_the_first(dtype):
    """Equal logits within a beam, equal beams, a constant vocabulary, a few
    values only: more equal candidates than any list holds."""
    torch = torch_cuda()
    rng = np.random.default_rng(7)
    for vocab in (50, 2049, 9000):
        few = torch.from_numpy(rng.integers(0, 3, (6, vocab)).astype(np.float32)).to(dtype_of(dtype)).cuda()
        _run(few, np.zeros((2, 3)))
        _run(few, np.zeros((2, 3)), 64 if vocab * 3 >= 64 else 3)
        _run(torch.zeros((6, vocab), dtype=dtype_of(dtype), device="cuda"), np.zeros((2, 3)), 20)
        signed = torch.where(few == 1, -0.0, 0.0).to(dtype_of(dtype))                  # -0 and 0 are equal
        _run(signed, np.zeros((2, 3)), 20)
    same = _logits(rng, 1, 4000, dtype).expand(4, 4000).contiguous()
    _run(same, np.full((1, 4), -1.0), 8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_vocabularies(dtype):
    """Nothing, one token, a few or all but a few allowed."""
    torch = torch_cuda()
    rng = np.random.default_rng(8)
    vocab = 6007
    for keep in ([], [17], [6006], [0, 1, 2], list(range(100, 140)), list(range(4000)), list(range(0, vocab, 2))):
        x = torch.full((6, vocab), -math.inf, dtype=dtype_of(dtype), device="cuda")
        if keep:
            x[:, keep] = _logits(rng, 6, len(keep), dtype)
        _run(x, -rng.random((2, 3)), 3)
        _run(x, -rng.random((2, 3)), 12)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [9000, 40001])          # 8 logits a lane, and 32
def test_candidates_in_few_lanes_and_in_all(dtype, vocab):
    """The best logits in some lanes of a wave only (tokens by their 16-byte
    grain), fewer and more of them than a list holds; few values; masks."""
    torch = torch_cuda()
    rng = np.random.default_rng(vocab)
    grain = 8 if dtype == "bf16" else 4
    lane = np.arange(vocab) // grain % 64
    base = rng.random((6, vocab))
    for lanes in (1, 3, 32, 33):
        x = np.where(lane < lanes, 10 + base, base)
        x[:, lane == 0] = np.minimum(x[:, lane == 0], 10.25)     # most of the other lanes' are above its maximum
        for n_out in (1, lanes, 64):
            _run(torch.from_numpy(x.astype(np.float32)).to(dtype_of(dtype)).cuda(), -rng.random((2, 3)), n_out)
    few = torch.from_numpy(rng.integers(0, 3, (6, vocab)).astype(np.float32)).to(dtype_of(dtype)).cuda()
    for n_out in (3, 40, 64):
        _run(few, np.zeros((2, 3)), n_out)
    for keep in ([], [vocab - 1], list(range(vocab - 70, vocab)), list(range(1, vocab, 2))):
        x = torch.full((6, vocab), -math.inf, dtype=dtype_of(dtype), device="cuda")
        if keep:
            x[:, keep] = _logits(rng, 6, len(keep), dtype)
        for n_out in (3, 40):
            _run(x, -rng.random((2, 3)), n_out)


def test_finished_first_and_hopeless_beams():
    torch = torch_cuda()
    rng = np.random.default_rng(9)
    x = _logits(rng, 12, 3001, "f32")
    first = np.full((3, 4), -np.inf)
    first[:, 0] = 0
    _run(x, first)                                        # a first step: one beam of each request
    _run(x, np.full((3, 4), -np.inf))                     # none at all
    done = rng.random((3, 4)) < 0.5
    done[0], done[1] = True, False
    for eos in (0, 2, 3000):
        _run(x, -12 * rng.random((3, 4)), None, done, eos)
        _run(x, -12 * rng.random((3, 4)), 9, done, eos)
        _run(x, first, 9, done, eos)
    _run(x, -rng.random((3, 4)), None, None, 2)
    odd = -rng.random((3, 4))
    odd[0, 1], odd[1, 2], odd[2, 0] = np.nan, -np.inf, np.inf
    _run(x, odd)
    _run(x, odd, 5, done, 1)
    for bad in (math.nan, math.inf):                      # logits that are no distribution
        y = x.clone()
        y[1, 2999], y[7, 0], y[8, :] = bad, bad, bad
        _run(y, -rng.random((3, 4)), 6)
        _run(y, -rng.random((3, 4)), 6, done, 1)
    huge = x.clone()
    huge[:, 5] = 3e38
    _run(huge, -rng.random((3, 4)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_at_any_stride_and_alignment(dtype):
    torch = torch_cuda()
    rng = np.random.default_rng(10)
    vocab = 4099
    x = _logits(rng, 8, vocab, dtype)
    scores = -rng.random((2, 4))
    for ld, off in ((vocab, 1), (vocab + 3, 0), (vocab + 5, 3), (2 * vocab, 7)):
        flat = torch.full((8 * ld + off + 16,), math.nan, dtype=x.dtype, device="cuda")   # nothing between rows is read
        view = flat[off:off + 8 * ld].view(8, ld)[:, :vocab]
        view.copy_(x)
        _run(view, scores, 6)
