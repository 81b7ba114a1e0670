"""GPU: how exactly fp32 attention forms its scores."""
import numpy as np
import pytest

from tests.gpu_common import torch_cuda
from tests.paged_common import ints

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("hd", [32, 64, 128])
def test_long_sums_of_one_sign(hd):
    """Two keys of one score S, as hd equal products a and as one product, with
    values 1 and -1: the output is tanh of half the scores' difference, and 0.
    The products are summed in four sums of n = hd / 4, each addition off by U of
    the sum so far, U S (n + 1) / 2 together, and the three sums of those are off
    by 2 U S; each score's product with log2 e by U S; the rest is U of 1.  The
    last bits of a make the additions of some binade err to the same side."""
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    a = np.array([1 + 2.0 ** -j + s * 2.0 ** -23 for j in range(15, 23) for s in (-1, 1, 3)], np.float32)
    k, v = np.zeros((len(a), 1, 2, hd), np.float32), np.zeros((len(a), 1, 2, hd), np.float32)
    k[:, 0, 0] = a[:, None]
    k[:, 0, 1, 0] = hd * a
    v[:, 0, 0], v[:, 0, 1] = 1, -1
    t = lambda x: torch.from_numpy(x).cuda()
    rows = len(a)
    got = paged.attention(t(np.ones((rows, 1, hd), np.float32)), t(k), t(v), ints(np.arange(rows)[:, None]),
                          ints(np.full(rows, 2)), scale=1.0)
    tol = ((hd / 4 + 1) / 2 + 2 + 2) * U * (hd * a.astype(np.float64)) / 2 + 4 * U
    err = np.abs(got[:, 0].double().cpu().numpy()).max(1)
    assert (err <= tol).all(), np.max(err / tol)
