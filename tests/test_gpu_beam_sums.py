"""GPU: how exactly beam selection's totals are formed.  With a score near lse -
maximum the best total is next to nothing, and shows the error of the lse."""
import numpy as np
import pytest

from tests.gpu_common import torch_cuda
from tests.paged_common import dtype_of, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [7, 500, 8000, 65537])
@pytest.mark.parametrize("scale", [1.0, 3.0, 6.0, 10.0, 40.0])
def test_the_error_of_a_total(dtype, vocab, scale):
    """Each power is off by 2^-23, by the rounding of maximum - logit (2^-24 of
    it) and of its product with log2 e (2^-24 of it), and seven roundings of a
    sum of eight follow; what comes then is in double.  The total is rounded
    once."""
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(vocab)
    x = torch.from_numpy((scale * rng.standard_normal((64, vocab))).astype(np.float32)).to(dtype_of(dtype)).cuda()
    v = host(x)
    d = v.max(1, keepdims=True) - v
    p = np.exp(-d)
    lse = v.max(1) + np.log(p.sum(1))
    mean = (p * d).sum(1) / p.sum(1)
    score = (lse - v.max(1)).astype(np.float32)
    got = host(paged.beam_select(x, torch.from_numpy(score[:, None]).cuda(), n_out=1)[2])[:, 0]
    want = score.astype(np.float64) - (lse - v.max(1))
    tol = (9 + 2 * mean) * 2.0 ** -24 + np.abs(want) * 2.0 ** -24 + np.abs(v).max(1) * 2.0 ** -51
    assert (np.abs(got - want) <= tol).all(), np.max(np.abs(got - want) / tol)
